// Rows of the paged key/value cache that change their places: the accepted path of a tree of drafts, and eviction by weight.
//
// Both move rows towards the front of their sequence, in order: the t-th row goes from place f(t) >= t (f ascending) to place t.  So the place that row t is
// written to can be the source of rows up to t only, never of later ones: once the rows up to t have been read, row t may be written.
#include "kv_attention.cuh"

namespace siso {
namespace kve {

using umma2::cluster_sync;

// The pages of all layers as bytes: `piece` = 16 or 8, which divides every row and stride
struct Pages {
    char *k, *v;
    uint8_t *k_exp, *v_exp;
    long long n_pages, stride_layer, stride_page, stride_token, stride_head;       // bytes
    int page_size, n_kv_heads, n_layers, pieces;                                   // pieces of a row
};
template <int PIECE> struct Bytes;
template <> struct Bytes<16> { using T = uint4; };
template <> struct Bytes<8> { using T = uint2; };

static Pages pages_of(const Kv *h, int &piece) {
    const siso_kv_config_t &g = h->cfg;
    const long long eb = kv_elem_bytes(g.dtype), row = g.head_dim * eb;
    Pages p;
    p.k = static_cast<char *>(g.d_k);
    p.v = static_cast<char *>(g.d_v);
    p.k_exp = g.d_k_exp;
    p.v_exp = g.d_v_exp;
    p.n_pages = g.n_pages;
    p.stride_layer = g.stride_layer * eb;
    p.stride_page = g.stride_page * eb;
    p.stride_token = g.stride_token * eb;
    p.stride_head = g.stride_head * eb;
    p.page_size = g.page_size;
    p.n_kv_heads = g.n_kv_heads;
    p.n_layers = g.n_layers;
    piece = ((row | p.stride_layer | p.stride_page | p.stride_token | p.stride_head) & 15) == 0 ? 16 : 8;
    p.pieces = static_cast<int>(row / piece);
    return p;
}

// ---- the accepted path ------------------------------------------------------------------------------------------------------
// A thread owns one piece (16 bytes) of the rows of one layer, head and side (K or V) and takes the path's rows in order, eight in flight; the
// places of up to KEEP rows are worked out by the CTA at a time.  Bound by latency: three dependent trips (path, page, row).  6 rows of 8 layers x 8 heads x 128
// bf16: 8 us; up to 12 rows of 48 sequences in 16 layers of 8-bit pages, 38 MB read and written: 11 to 14 us.
constexpr int KEEP_THREADS = 256, KEEP = 64, KEEP_U = 8;

struct KeepArgs {
    Pages p;
    const int32_t *path, *accepted, *cu_q, *kv_len, *pages;
    long long pages_stride;
    int32_t *new_len;
    kva::FastDiv by_page, by_pieces;
    int max_path, max_pages, items;              // items: pieces and exponents of one layer and token
    int *status;
};

template <int PIECE>
__global__ void __launch_bounds__(KEEP_THREADS)
keep_path_kernel(const __grid_constant__ KeepArgs g) {
    using T = typename Bytes<PIECE>::T;
    __shared__ int32_t page[2][KEEP], tok[2][KEEP];           // where a row comes from and goes to; page -1: it stays
    wait_for_earlier();
    dependents_may_start();
    const int b = blockIdx.x, layer = blockIdx.y;
    const int32_t *path = g.path + static_cast<long long>(b) * g.max_path;
    // the entries of a block of the path, asked for before it is known how many count
    int node = 0, earlier = 0;
    auto look_up = [&](int t) {
        if (threadIdx.x < KEEP && t < g.max_path) {
            node = path[t];
            earlier = t > 0 ? path[t - 1] : 0;
        }
    };
    look_up(threadIdx.x);
    const long long cap = static_cast<long long>(g.max_pages) * g.p.page_size;
    const int len = static_cast<int>(min(static_cast<long long>(max(g.kv_len[b], 0)), cap));
    const int n_q = max(0, g.cu_q[b + 1] - g.cu_q[b]), before = len - n_q;
    const bool first = layer == 0 && blockIdx.z == 0;
    const int wanted = before < 0 ? 0 : min(max(g.accepted[b], 0), g.max_path);
    bool bad = before < 0 && n_q > 0;
    int done = 0;
    for (int t0 = 0; t0 < wanted && !bad; t0 += KEEP) {
        // the entry t of the path goes on with it if it is a node behind the entry before
        const int t = t0 + threadIdx.x;
        bool fine = true;
        if (threadIdx.x < KEEP && t < wanted) {
            fine = node > max(earlier, 0) && node < n_q;
            page[0][threadIdx.x] = page[1][threadIdx.x] = -1;
            if (fine && node != t + 1) {
                const int from = before + node, to = before + 1 + t;
                const int i0 = static_cast<int>(g.by_page.div(static_cast<uint32_t>(from))), i1 = static_cast<int>(g.by_page.div(static_cast<uint32_t>(to)));
                const int p0 = g.pages[b * g.pages_stride + i0], p1 = g.pages[b * g.pages_stride + i1];
                if (p0 >= 0 && p0 < g.p.n_pages && p1 >= 0 && p1 < g.p.n_pages) {
                    page[0][threadIdx.x] = p0;
                    page[1][threadIdx.x] = p1;
                    tok[0][threadIdx.x] = from - i0 * g.p.page_size;
                    tok[1][threadIdx.x] = to - i1 * g.p.page_size;
                } else if (first) set_status(g.status, SISO_ERR_INVALID_ARG);
            }
        }
        // how many entries of these go on: up to the first that does not (warps 0 and 1 hold them)
        __shared__ uint32_t broken[2];
        const uint32_t out = __ballot_sync(0xFFFFFFFFu, !fine);
        if (threadIdx.x < KEEP && (threadIdx.x & 31) == 0) broken[threadIdx.x >> 5] = out;
        __syncthreads();
        int n = min(KEEP, wanted - t0);
        if (broken[0] | broken[1]) {
            bad = true;
            n = broken[0] ? __ffs(broken[0]) - 1 : 32 + __ffs(broken[1]) - 1;
        }
        for (int item = blockIdx.z * KEEP_THREADS + threadIdx.x; item < g.items; item += gridDim.z * KEEP_THREADS) {
            const int rows = 2 * g.p.n_kv_heads, n_pieces = rows * g.p.pieces;
            if (item < n_pieces) {
                const int row = static_cast<int>(g.by_pieces.div(static_cast<uint32_t>(item))), head = row >> 1;
                char *base = ((row & 1) ? g.p.v : g.p.k) + layer * g.p.stride_layer + head * g.p.stride_head + (item - row * g.p.pieces) * PIECE;
                for (int t1 = 0; t1 < n; t1 += KEEP_U) {
                    T x[KEEP_U];
#pragma unroll
                    for (int u = 0; u < KEEP_U; ++u)
                        if (t1 + u < n && page[0][t1 + u] >= 0)
                            x[u] = *reinterpret_cast<const T *>(base + page[0][t1 + u] * g.p.stride_page + tok[0][t1 + u] * g.p.stride_token);
#pragma unroll
                    for (int u = 0; u < KEEP_U; ++u)
                        if (t1 + u < n && page[0][t1 + u] >= 0)
                            *reinterpret_cast<T *>(base + page[1][t1 + u] * g.p.stride_page + tok[1][t1 + u] * g.p.stride_token) = x[u];
                }
            } else {                                          // an exponent
                const int row = item - n_pieces, head = row >> 1;
                uint8_t *base = (row & 1) ? g.p.v_exp : g.p.k_exp;
                const long long at = static_cast<long long>(layer) * g.p.n_pages;
                for (int t1 = 0; t1 < n; ++t1)
                    if (page[0][t1] >= 0)
                        base[((at + page[1][t1]) * g.p.n_kv_heads + head) * g.p.page_size + tok[1][t1]] =
                            base[((at + page[0][t1]) * g.p.n_kv_heads + head) * g.p.page_size + tok[0][t1]];
            }
        }
        done += n;
        look_up(t + KEEP);
        __syncthreads();
    }
    if (first && threadIdx.x == 0) {
        g.new_len[b] = n_q > 0 && before >= 0 ? before + 1 + done : len;
        if (bad) set_status(g.status, SISO_ERR_INVALID_ARG);
    }
}

// ---- eviction ---------------------------------------------------------------------------------------------------------------
// A cluster of CTAs per (layer, sequence, kv head).  Weights become whole numbers of the same order, and the smallest weight that stays is found eight bits at a time
// from counts of the numbers' digits.  The places that stay are listed in order, then the rows are moved in waves: all CTAs read a wave's rows into
// registers, meet, and write them, which is safe in place because of the order (see above).
constexpr int THREADS = 512, WARPS = THREADS / 32, U = 8;        // U: pieces of a thread in flight
constexpr int R = 16, KEYS = 40 * 1024;           // weights that a thread keeps in registers; that a CTA keeps in shared memory
// Which places stay is found out by each CTA of the cluster from all weights (up to 8192), so that none waits for another's counts (24 sequences of up to 4200 tokens: 31 us
// and 37 us); or each has a part of the weights, in registers (16,385 tokens: 31 us and 35 us) or, above 65,536, in shared memory as far as they fit, and the counts are exchanged.
// Bound by latency up to the rows: weights, digits, list and places are trips and barriers one after another; the rows then go at bandwidth.  Now measured: 16,385 to 2048
// tokens, four layers x 8 heads x 128 bf16, 35 us, about 10 of them for the rows; 24 sequences of 1100 to 4200 tokens to 1000, two layers x 4 heads x 64 e4m3, 28 us; in place
// 42 and 29 us, as all CTAs of a cluster meet between reading and writing a wave (inputs not in L2).
enum Mode { ALONE, SHARED_REGS, SHARED };
constexpr int SLOTS = 1024;                       // rows of a CTA whose places are worked out at a time

struct EvictArgs {
    Pages p;
    float *weights;                               // [layers, pages, kv heads, page_size]
    const int32_t *kv_len, *pages, *out_pages;
    long long pages_stride, out_stride;
    int32_t *new_len, *kept;
    kva::FastDiv by_page;
    int max_pages, out_max_pages, n_seqs, budget, recent, keys;
    int *status;
};
// a number that orders as the weight does: NaN 0, -infinity 0x007FFFFF, 0 and -0 0x80000000
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t x = __float_as_uint(w + 0.f);
    return w != w ? 0u : (x & 0x80000000u) ? ~x : x | 0x80000000u;
}
// The same word of shared memory in CTA `rank` of the cluster: added to, written
__device__ __forceinline__ uint32_t address_in(const uint32_t *p, uint32_t rank) {
    return umma2::cluster_addr(static_cast<uint32_t>(__cvta_generic_to_shared(p)), rank);
}
__device__ __forceinline__ void add_in(uint32_t *p, uint32_t rank, uint32_t x) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(address_in(p, rank)), "r"(x) : "memory");
}
__device__ __forceinline__ void put_in(uint32_t *p, uint32_t rank, uint32_t x) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(address_in(p, rank)), "r"(x) : "memory");
}
// counts of a digit lie so that a lane's eight neighbouring digits are in its own bank
__device__ __forceinline__ int place_of(uint32_t digit) { return static_cast<int>((digit & 7u) * 32u + (digit >> 3)); }
// From the top digit down, where the wanted-th number lies: (digit, how many are in larger ones, how many in it).  For every warp by itself
__device__ __forceinline__ uint3 find_digit(const uint32_t *counts, uint32_t wanted, int lane) {
    uint32_t mine[8], total = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) { mine[i] = counts[(7 - i) * 32 + 31 - lane]; total += mine[i]; }
    uint32_t upto = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += y;
    }
    const int from = max(__ffs(__ballot_sync(0xFFFFFFFFu, upto >= wanted)) - 1, 0);
    uint32_t before = upto - total, digit = 0u, larger = 0u, here = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (before < wanted) { digit = 255u - (lane * 8 + i); larger = before; here = mine[i]; }
        before += mine[i];
    }
    return make_uint3(__shfl_sync(0xFFFFFFFFu, digit, from), __shfl_sync(0xFFFFFFFFu, larger, from), __shfl_sync(0xFFFFFFFFu, here, from));
}

template <int PIECE, int MODE>
__global__ void __launch_bounds__(THREADS, 2)
evict_kernel(const __grid_constant__ EvictArgs g) {
    using T = typename Bytes<PIECE>::T;
    constexpr bool BY_ITSELF = MODE == ALONE, REGS = MODE != SHARED;
    extern __shared__ uint32_t keys[];
    uint16_t *list = reinterpret_cast<uint16_t *>(keys);          // BY_ITSELF: the places that stay
    __shared__ uint32_t hist[4][256], sums[BY_ITSELF ? 1 : 4][256];   // counts of this CTA, of all
    __shared__ uint32_t counts[2][8], warp_gt[WARPS], warp_eq[WARPS];
    __shared__ int4 moves[SLOTS];                 // page and token that a row comes from, that it goes to; page -1: it is not moved
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t rank, n_ctas;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    wait_for_earlier();
    dependents_may_start();
    const unsigned seg = blockIdx.x / n_ctas;
    const int head = static_cast<int>(seg % g.p.n_kv_heads);
    const int b = static_cast<int>(seg / g.p.n_kv_heads % g.n_seqs), layer = static_cast<int>(seg / g.p.n_kv_heads / g.n_seqs);
    const int page_size = g.p.page_size;
    const int32_t *pages = g.pages + b * g.pages_stride, *out_pages = g.out_pages + b * g.out_stride;
    const int len = static_cast<int>(min(static_cast<long long>(max(g.kv_len[b], 0)), static_cast<long long>(g.max_pages) * page_size));
    const int n_kept = min(len, g.budget);
    int32_t *kept = g.kept + static_cast<long long>(seg) * g.budget;
    // of weights and exponents: row (page, token) of this layer and head
    const long long small0 = (static_cast<long long>(layer) * g.p.n_pages * g.p.n_kv_heads + head) * page_size, small_page = static_cast<long long>(g.p.n_kv_heads) * page_size;
    auto in_pool = [&](int p) { return p >= 0 && p < g.p.n_pages; };
    auto together = [&]() {
        if (n_ctas > 1) cluster_sync();
        else __syncthreads();
    };

    if (layer == 0 && head == 0 && rank == 0 && threadIdx.x == 0) g.new_len[b] = n_kept;
    const int step = static_cast<int>(n_ctas) * THREADS, me = static_cast<int>(rank) * THREADS + threadIdx.x;
    for (int t = n_kept + me; t < g.budget; t += step) kept[t] = -1;
    const int cand = len - g.recent, wanted = g.budget - g.recent;
    for (int t = (len <= g.budget ? 0 : wanted) + me; t < n_kept; t += step) kept[t] = len <= g.budget ? t : cand + t - wanted;
    if constexpr (BY_ITSELF)
        if (len > g.budget)
            for (int t = wanted + static_cast<int>(threadIdx.x); t < n_kept; t += THREADS) list[t] = static_cast<uint16_t>(cand + t - wanted);
    auto place_kept = [&](int t) { return BY_ITSELF ? (len <= g.budget ? t : static_cast<int>(list[t])) : kept[t]; };
    if (len > g.budget && wanted > 0) {           // (cand > wanted)
        // each CTA has a part of the places, each warp a part of it
        const int parts = BY_ITSELF ? WARPS : static_cast<int>(n_ctas) * WARPS, warp_each = ((cand + parts - 1) / parts + 31) & ~31, each = warp_each * WARPS;
        const int lo = BY_ITSELF ? 0 : static_cast<int>(min(static_cast<long long>(rank) * each, static_cast<long long>(cand))), hi = static_cast<int>(min(static_cast<long long>(lo) + each, static_cast<long long>(cand)));
        const int w_lo = static_cast<int>(min(static_cast<long long>(lo) + warp * warp_each, static_cast<long long>(hi))),
                  w_hi = static_cast<int>(min(static_cast<long long>(w_lo) + warp_each, static_cast<long long>(hi)));
        uint32_t mine[REGS ? R : 1];
        auto look_up = [&](int i) {
            const int at = static_cast<int>(g.by_page.div(static_cast<uint32_t>(i))), p = pages[at];
            if (!in_pool(p)) { set_status(g.status, SISO_ERR_INVALID_ARG); return 0u; }
            return order_of(g.weights[small0 + p * small_page + i - at * page_size]);
        };
        // f(place, its number, whether there is one) for 32 neighbours at a time, in order
        auto for_each = [&](auto f) __attribute__((always_inline)) {
            if constexpr (REGS) {
#pragma unroll
                for (int k = 0; k < R; ++k)
                    if (w_lo + 32 * k < w_hi) f(w_lo + 32 * k + lane, mine[k], w_lo + 32 * k + lane < w_hi);
            } else {
                for (int i = w_lo + lane; i - lane < w_hi; i += 32)
                    f(i, i >= w_hi ? 0u : i - lo < g.keys ? keys[i - lo] : look_up(i), i < w_hi);
            }
        };
        for (int i = threadIdx.x; i < 4 * 256; i += THREADS) {
            (&hist[0][0])[i] = 0u;
            if constexpr (!BY_ITSELF) (&sums[0][0])[i] = 0u;
        }
        if constexpr (REGS) {                         // all of a thread's weights in flight: their pages, then they
            // (no branches: a load that hangs on one waits for the one before it)
            bool bad = false;
            int p[R];
#pragma unroll
            for (int k = 0; k < R; ++k) p[k] = pages[g.by_page.div(static_cast<uint32_t>(min(w_lo + 32 * k + lane, cand - 1)))];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int i = min(w_lo + 32 * k + lane, cand - 1), t = i - static_cast<int>(g.by_page.div(static_cast<uint32_t>(i))) * page_size;
                mine[k] = __float_as_uint(g.weights[small0 + (in_pool(p[k]) ? p[k] : 0) * small_page + t]);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                bad = bad || !in_pool(p[k]);
                mine[k] = in_pool(p[k]) ? order_of(__uint_as_float(mine[k])) : 0u;
            }
            if (bad) set_status(g.status, SISO_ERR_INVALID_ARG);
        } else {
            for (int i = w_lo + lane; i < w_hi && i - lo < g.keys; i += 32) keys[i - lo] = look_up(i);
        }
        if constexpr (BY_ITSELF) __syncthreads();
        else together();                              // (no CTA adds to another's counts before it has cleared them)
        // the wanted-th largest: `least`, of which `ties` are wanted
        uint32_t least = 0u;
        int ties = wanted;
        for (int pass = 0;; ++pass) {
            const int shift = 24 - 8 * pass;
            uint32_t *h = hist[pass];
            for_each([&](int, uint32_t x, bool there) {
                if (there && (pass == 0 || x >> (shift + 8) == least >> (shift + 8))) atomicAdd(&h[place_of((x >> shift) & 255u)], 1u);
            });
            // each CTA adds its counts to those of all: nothing is read from afar, the barrier sees to the rest
            __syncthreads();
            if (!BY_ITSELF && n_ctas > 1) {
                if (threadIdx.x < 256) {
                    const uint32_t n = h[threadIdx.x];
                    if (n)
                        for (uint32_t c = 0; c < n_ctas; ++c) add_in(&sums[BY_ITSELF ? 0 : pass][threadIdx.x], c, n);
                }
                cluster_sync();
                h = sums[BY_ITSELF ? 0 : pass];
            }
            const uint3 d = find_digit(h, static_cast<uint32_t>(ties), lane);
            least |= d.x << shift;
            ties -= static_cast<int>(d.y);
            if (shift == 0) break;
            if (static_cast<uint32_t>(ties) == d.z) {            // all of this digit stay: what is larger than the number before its first
                least -= 1u;
                ties = 0;
                break;
            }
        }
        // how many of each warp's places are heavier, and as heavy; how many before them
        uint32_t gt = 0u, eq = 0u;
        for_each([&](int, uint32_t x, bool there) {
            gt += __popc(__ballot_sync(0xFFFFFFFFu, there && x > least));
            eq += __popc(__ballot_sync(0xFFFFFFFFu, there && x == least));
        });
        if (lane == 0) { warp_gt[warp] = gt; warp_eq[warp] = eq; }
        __syncthreads();
        uint32_t w_gt = lane < WARPS ? warp_gt[lane] : 0u, w_eq = lane < WARPS ? warp_eq[lane] : 0u;
        gt = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? w_gt : 0u);
        eq = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? w_eq : 0u);
        if (!BY_ITSELF && n_ctas > 1) {
            w_gt = __reduce_add_sync(0xFFFFFFFFu, w_gt);
            w_eq = __reduce_add_sync(0xFFFFFFFFu, w_eq);
            if (threadIdx.x < n_ctas) { put_in(&counts[0][rank], threadIdx.x, w_gt); put_in(&counts[1][rank], threadIdx.x, w_eq); }
            cluster_sync();
            for (uint32_t c = 0; c < rank; ++c) { gt += counts[0][c]; eq += counts[1][c]; }
        }
        // their places in the list, in order
        for_each([&](int i, uint32_t x, bool there) {
            const bool more = there && x > least, same = there && x == least;
            const uint32_t is_gt = __ballot_sync(0xFFFFFFFFu, more), is_eq = __ballot_sync(0xFFFFFFFFu, same), below = (1u << lane) - 1u;
            const uint32_t my_gt = gt + __popc(is_gt & below), my_eq = eq + __popc(is_eq & below);
            // (the bound holds unless weights change meanwhile, as where sequences share pages)
            const uint32_t to = my_gt + min(my_eq, static_cast<uint32_t>(ties));
            if ((more || (same && my_eq < static_cast<uint32_t>(ties))) && to < static_cast<uint32_t>(wanted)) {
                if constexpr (BY_ITSELF) list[to] = static_cast<uint16_t>(i);
                else kept[to] = i;
            }
            gt += __popc(is_gt);
            eq += __popc(is_eq);
        });
    }
    // whether any row may be written to a place that another row is read from
    bool same_page = false;
    for (int i = threadIdx.x; i < g.out_max_pages && static_cast<long long>(i) * page_size < n_kept; i += THREADS)
        same_page = same_page || (i < g.max_pages && out_pages[i] == pages[i]);
    const bool in_place = __syncthreads_or(same_page) != 0;
    if constexpr (BY_ITSELF) {
        if (len > g.budget)
            for (int t = me; t < wanted; t += step) kept[t] = list[t];
    } else {
        __threadfence();
        together();
    }

    // ---- the rows move, in waves of cta_wave tokens of each CTA, the CTAs' one after the other
    // tokens that the CTA takes side by side: no more than leave it a thread for the places of each of U times as many
    const int per_token = 2 * g.p.pieces, tokens_step = min(THREADS / per_token, THREADS / U), cta_wave = tokens_step * U, wave = cta_wave * static_cast<int>(n_ctas);
    const int waves = SLOTS / cta_wave;           // whose places are worked out at a time
    const int off = static_cast<int>(threadIdx.x) / per_token, item = static_cast<int>(threadIdx.x) - off * per_token;
    const bool is_v = item >= g.p.pieces;
    char *base = (is_v ? g.p.v : g.p.k) + layer * g.p.stride_layer + head * g.p.stride_head + (is_v ? item - g.p.pieces : item) * PIECE;
    for (int w0 = 0; w0 < n_kept; w0 += waves * wave) {
        // where the CTA's tokens of these waves come from and go to; their weights and exponents, which are written once all CTAs have read theirs
        long long small_to[SLOTS / THREADS];
        float weight[SLOTS / THREADS];
        uint32_t exps[SLOTS / THREADS];
#pragma unroll
        for (int x = 0; x < SLOTS / THREADS; ++x) {
            const int slot = x * THREADS + static_cast<int>(threadIdx.x), nth = slot / cta_wave, t = w0 + nth * wave + static_cast<int>(rank) * cta_wave + slot - nth * cta_wave;
            small_to[x] = -1;
            int4 m = make_int4(-1, 0, 0, 0);
            if (nth < waves && t < n_kept) {
                const int j = place_kept(t);
                if (j >= t && j < len) {                                          // (always, unless sequences share pages, see above)
                    const int i0 = static_cast<int>(g.by_page.div(static_cast<uint32_t>(j))), i1 = static_cast<int>(g.by_page.div(static_cast<uint32_t>(t)));
                    const int p0 = pages[i0], p1 = i1 < g.out_max_pages ? out_pages[i1] : -1;
                    if (!in_pool(p0) || !in_pool(p1)) set_status(g.status, SISO_ERR_INVALID_ARG);
                    else if (p0 != p1 || j - i0 * page_size != t - i1 * page_size) m = make_int4(p0, j - i0 * page_size, p1, t - i1 * page_size);
                }
            }
            moves[slot] = m;
            if (m.x >= 0) {
                const long long from = small0 + m.x * small_page + m.y;
                small_to[x] = small0 + m.z * small_page + m.w;
                weight[x] = g.weights[from];
                if (g.p.k_exp) exps[x] = g.p.k_exp[from] | static_cast<uint32_t>(g.p.v_exp[from]) << 8;
            }
        }
        __syncthreads();
        for (int nth = 0; nth < waves && w0 + nth * wave < n_kept; ++nth) {
            const int4 *here = moves + nth * cta_wave + off;
            T x[U];
            if (off < tokens_step)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int4 m = here[u * tokens_step];
                    if (m.x >= 0) x[u] = *reinterpret_cast<const T *>(base + m.x * g.p.stride_page + m.y * g.p.stride_token);
                }
            if (in_place) together();
            if (off < tokens_step)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int4 m = here[u * tokens_step];
                    if (m.x >= 0) *reinterpret_cast<T *>(base + m.z * g.p.stride_page + m.w * g.p.stride_token) = x[u];
                }
            if (nth == 0)
#pragma unroll
                for (int y = 0; y < SLOTS / THREADS; ++y)
                    if (small_to[y] >= 0) {
                        g.weights[small_to[y]] = weight[y];
                        if (g.p.k_exp) { g.p.k_exp[small_to[y]] = static_cast<uint8_t>(exps[y]); g.p.v_exp[small_to[y]] = static_cast<uint8_t>(exps[y] >> 8); }
                    }
        }
        __syncthreads();                          // (`moves` is read until here)
    }
}

template <int PIECE> static siso_status_t run_evict(Kv *h, const EvictArgs &g0, int max_cand, cudaStream_t s) {
    EvictArgs g = g0;
    const long long segs = static_cast<long long>(g.p.n_layers) * g.n_seqs * g.p.n_kv_heads;
    const bool alone = max_cand <= THREADS * R && max_cand + g.recent <= 65536;      // (places in 2 bytes)
    // as many CTAs for each as run at once (two per SM), or, where they share the weights, up to twice that
    const long long room = 2ll * h->sm_count;
    int ctas = 1;
    while (ctas < 8 && (segs * ctas * 2 <= (alone ? room : 2 * room) || (!alone && max_cand > ctas * THREADS * R))) ctas *= 2;
    if (segs * ctas >= (1ll << 31)) return SISO_ERR_UNSUPPORTED;
    const bool regs = max_cand <= ctas * THREADS * R;
    const int each = ((max_cand + ctas * WARPS - 1) / (ctas * WARPS) + 31) / 32 * 32 * WARPS;
    g.keys = std::min(KEYS, each);
    const size_t smem = alone ? (static_cast<size_t>(std::min(g.budget, max_cand + g.recent)) * 2 + 15) / 16 * 16 : regs ? 0 : static_cast<size_t>(g.keys) * 4;
    auto *kernel = alone ? evict_kernel<PIECE, ALONE> : regs ? evict_kernel<PIECE, SHARED_REGS> : evict_kernel<PIECE, SHARED>;
    const uint32_t bit = 1u << (alone ? 16 : 17);
    if ((alone || !regs) && !(h->attr_set & bit)) {
        SISO_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, alone ? 65536 * 2 : KEYS * 4));
        h->attr_set |= bit;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(segs * ctas));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // (as launch_early)
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    SISO_CUDA(cudaLaunchKernelEx(&cfg, kernel, g));
    return SISO_OK;
}

}  // namespace kve
}  // namespace siso

using namespace siso;

extern "C" siso_status_t siso_kv_keep_path(siso_kv_t *h, const int32_t *d_path, const int32_t *d_accepted, int32_t max_path, const int32_t *d_cu_q,
                                           const int32_t *d_kv_len, const int32_t *d_pages, int64_t pages_stride, int32_t max_pages,
                                           int32_t n_seqs, int32_t *d_new_len, void *stream) {
    if (!h || max_path < 0 || max_pages < 0 || n_seqs < 0 || pages_stride < 0) return SISO_ERR_INVALID_ARG;
    if (n_seqs == 0) return SISO_OK;
    if ((max_path > 0 && !d_path) || !d_accepted || !d_cu_q || !d_kv_len || (max_pages > 0 && !d_pages) || !d_new_len || d_new_len == d_kv_len)
        return SISO_ERR_INVALID_ARG;
    if (static_cast<int64_t>(max_pages) * h->cfg.page_size >= (1ll << 31) - 65536 || h->cfg.n_layers > 65535) return SISO_ERR_UNSUPPORTED;
    const OnDevice on(h->cfg.device);
    SISO_CUDA(on.error());
    int piece;
    kve::KeepArgs g;
    g.p = kve::pages_of(h, piece);
    g.path = d_path;
    g.accepted = d_accepted;
    g.cu_q = d_cu_q;
    g.kv_len = d_kv_len;
    g.pages = d_pages;
    g.pages_stride = pages_stride;
    g.new_len = d_new_len;
    g.max_path = max_path;
    g.max_pages = max_pages;
    g.by_page.set(static_cast<uint32_t>(h->cfg.page_size));
    g.by_pieces.set(static_cast<uint32_t>(g.p.pieces));
    g.items = 2 * g.p.n_kv_heads * (g.p.pieces + (g.p.k_exp ? 1 : 0));
    g.status = h->status;
    const int z = std::min(64, (g.items + kve::KEEP_THREADS - 1) / kve::KEEP_THREADS);
    const dim3 grid(static_cast<unsigned>(n_seqs), static_cast<unsigned>(g.p.n_layers), static_cast<unsigned>(z));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return launch_early(piece == 16 ? kve::keep_path_kernel<16> : kve::keep_path_kernel<8>, grid, kve::KEEP_THREADS, 0, s, g);
}

extern "C" siso_status_t siso_kv_evict(siso_kv_t *h, float *d_weights, const int32_t *d_kv_len, const int32_t *d_pages, int64_t pages_stride,
                                       int32_t max_pages, const int32_t *d_out_pages, int64_t out_pages_stride, int32_t out_max_pages,
                                       int32_t n_seqs, int32_t budget, int32_t recent, int32_t *d_new_len, int32_t *d_kept, void *stream) {
    if (!h || max_pages < 0 || out_max_pages < 0 || n_seqs < 0 || pages_stride < 0 || out_pages_stride < 0) return SISO_ERR_INVALID_ARG;
    if (budget < 1 || recent < 0 || recent > budget) return SISO_ERR_INVALID_ARG;
    if (n_seqs == 0) return SISO_OK;
    if (!d_weights || !d_kv_len || (max_pages > 0 && !d_pages) || (out_max_pages > 0 && !d_out_pages) || !d_new_len || !d_kept || d_new_len == d_kv_len)
        return SISO_ERR_INVALID_ARG;
    const int64_t cap = static_cast<int64_t>(max_pages) * h->cfg.page_size;
    if (cap >= (1ll << 31) - 65536 || static_cast<int64_t>(out_max_pages) * h->cfg.page_size >= (1ll << 31) - 65536) return SISO_ERR_UNSUPPORTED;
    if (budget >= (1 << 30)) return SISO_ERR_UNSUPPORTED;
    const OnDevice on(h->cfg.device);
    SISO_CUDA(on.error());
    int piece;
    kve::EvictArgs g;
    g.p = kve::pages_of(h, piece);
    g.weights = d_weights;
    g.kv_len = d_kv_len;
    g.pages = d_pages;
    g.out_pages = d_out_pages;
    g.pages_stride = pages_stride;
    g.out_stride = out_pages_stride;
    g.new_len = d_new_len;
    g.kept = d_kept;
    g.max_pages = max_pages;
    g.out_max_pages = out_max_pages;
    g.n_seqs = n_seqs;
    g.budget = budget;
    g.recent = recent;
    g.by_page.set(static_cast<uint32_t>(h->cfg.page_size));
    g.status = h->status;
    const int max_cand = static_cast<int>(std::max<int64_t>(1, cap - recent));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return piece == 16 ? kve::run_evict<16>(h, g, max_cand, s) : kve::run_evict<8>(h, g, max_cand, s);
}
