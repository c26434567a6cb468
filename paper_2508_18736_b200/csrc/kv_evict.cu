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
// places of up to KEEP rows are worked out by the CTA at a time.  Bound by latency: three dependent trips (path, page, row).
constexpr int KEEP_THREADS = 256, KEEP = 64, KEEP_U = 8;

struct KeepArgs {
    Pages p;
    const int32_t *path, *accepted, *cu_q, *kv_len, *pages;
    long long pages_stride;
    int32_t *new_len;
    int max_path, max_pages, items;              // items: pieces and exponents of one layer and token
    int *status;
};

template <int PIECE>
__global__ void __launch_bounds__(KEEP_THREADS)
keep_path_kernel(const __grid_constant__ KeepArgs g) {
    using T = typename Bytes<PIECE>::T;
    __shared__ int32_t page[2][KEEP], tok[2][KEEP];           // where a row comes from and goes to; page -1: it stays
    const int b = blockIdx.x, layer = blockIdx.y;
    const long long cap = static_cast<long long>(g.max_pages) * g.p.page_size;
    const int len = static_cast<int>(min(static_cast<long long>(max(g.kv_len[b], 0)), cap));
    const int n_q = max(0, g.cu_q[b + 1] - g.cu_q[b]), before = len - n_q;
    const int32_t *path = g.path + static_cast<long long>(b) * g.max_path;
    const bool first = layer == 0 && blockIdx.z == 0;
    const int wanted = before < 0 ? 0 : min(max(g.accepted[b], 0), g.max_path);
    bool bad = before < 0 && n_q > 0;
    int done = 0;
    for (int t0 = 0; t0 < wanted && !bad; t0 += KEEP) {
        // the entry t of the path goes on with it if it is a node behind the entry before
        const int t = t0 + threadIdx.x;
        bool fine = true;
        if (threadIdx.x < KEEP && t < wanted) {
            const int node = path[t], earlier = t > 0 ? path[t - 1] : 0;
            fine = node > earlier && node < n_q;
            page[0][threadIdx.x] = page[1][threadIdx.x] = -1;
            if (fine && node != t + 1) {
                const int from = before + node, to = before + 1 + t;
                const int i0 = from / g.p.page_size, i1 = to / g.p.page_size;
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
                const int row = item / g.p.pieces, head = row >> 1;
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
        __syncthreads();
    }
    if (first && threadIdx.x == 0) {
        g.new_len[b] = n_q > 0 && before >= 0 ? before + 1 + done : len;
        if (bad) set_status(g.status, SISO_ERR_INVALID_ARG);
    }
}

// ---- eviction ---------------------------------------------------------------------------------------------------------------
// A cluster of CTAs per (layer, sequence, kv head).  Weights become whole numbers of the same order, each CTA keeps those of its part of the places in
// shared memory (as far as they fit), and the smallest weight that stays is found eight bits at a time from counts that the CTAs exchange.
// The places that stay are listed in order (d_kept, an output anyway), then the rows are moved in waves: all CTAs read a wave's rows into
// registers, meet, and write them, which is safe in place because of the order (see above).
constexpr int THREADS = 512, WARPS = THREADS / 32, U = 8, KEYS = 40 * 1024;      // KEYS: weights that a CTA keeps in shared memory

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
template <typename T> __device__ __forceinline__ T remote(const T *p, uint32_t rank) {
    uint32_t there, x;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(there) : "memory");
    return static_cast<T>(x);
}

// From the top digit down, where the wanted-th number lies: (digit, how many are in larger ones, how many in it).  For every warp by itself
__device__ __forceinline__ uint3 find_digit(const uint32_t *counts, uint32_t wanted, int lane) {
    uint32_t mine[8], total = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) { mine[i] = counts[255 - (lane * 8 + i)]; total += mine[i]; }
    uint32_t upto = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += y;
    }
    uint32_t before = upto - total, digit = 0u, larger = 0u, here = 0u;
    bool found = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (before < wanted && before + mine[i] >= wanted) { digit = 255u - (lane * 8 + i); larger = before; here = mine[i]; found = true; }
        before += mine[i];
    }
    const int from = max(__ffs(__ballot_sync(0xFFFFFFFFu, found)) - 1, 0);
    return make_uint3(__shfl_sync(0xFFFFFFFFu, digit, from), __shfl_sync(0xFFFFFFFFu, larger, from), __shfl_sync(0xFFFFFFFFu, here, from));
}

template <int PIECE>
__global__ void __launch_bounds__(THREADS, 2)
evict_kernel(const __grid_constant__ EvictArgs g) {
    using T = typename Bytes<PIECE>::T;
    extern __shared__ uint32_t keys[];
    __shared__ uint32_t hist[4][256], sums[2][256], counts[2], warp_gt[WARPS], warp_eq[WARPS];
    __shared__ int4 moves[THREADS];               // page and token that a row comes from, that it goes to; page -1: it is not moved
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t rank, n_ctas;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    const unsigned seg = blockIdx.x / n_ctas;
    const int head = static_cast<int>(seg % g.p.n_kv_heads);
    const int b = static_cast<int>(seg / g.p.n_kv_heads % g.n_seqs), layer = static_cast<int>(seg / g.p.n_kv_heads / g.n_seqs);
    const int page_size = g.p.page_size;
    const int32_t *pages = g.pages + b * g.pages_stride, *out_pages = g.out_pages + b * g.out_stride;
    const long long first_page = static_cast<long long>(layer) * g.p.n_pages;
    const int len = static_cast<int>(min(static_cast<long long>(max(g.kv_len[b], 0)), static_cast<long long>(g.max_pages) * page_size));
    const int n_kept = min(len, g.budget);
    int32_t *kept = g.kept + static_cast<long long>(seg) * g.budget;
    auto in_pool = [&](int p) { return p >= 0 && p < g.p.n_pages; };
    auto small_at = [&](int p, int t) { return ((first_page + p) * g.p.n_kv_heads + head) * page_size + t; };       // of weights and exponents
    auto together = [&]() {
        if (n_ctas > 1) cluster_sync();
        else __syncthreads();
    };

    if (layer == 0 && head == 0 && rank == 0 && threadIdx.x == 0) g.new_len[b] = n_kept;
    const int step = static_cast<int>(n_ctas) * THREADS, me = static_cast<int>(rank) * THREADS + threadIdx.x;
    for (int t = n_kept + me; t < g.budget; t += step) kept[t] = -1;
    if (len <= g.budget) {
        for (int t = me; t < n_kept; t += step) kept[t] = t;
    } else {
        const int cand = len - g.recent, wanted = g.budget - g.recent;         // (cand > wanted)
        for (int i = me; i < g.recent; i += step) kept[wanted + i] = cand + i;
        const int each = ((cand + static_cast<int>(n_ctas) - 1) / static_cast<int>(n_ctas) + WARPS * 32 - 1) / (WARPS * 32) * (WARPS * 32);
        const int lo = static_cast<int>(min(static_cast<long long>(rank) * each, static_cast<long long>(cand))), hi = min(cand, lo + each);
        auto look_up = [&](int i) {
            const int at = static_cast<int>(g.by_page.div(static_cast<uint32_t>(i))), p = pages[at];
            return in_pool(p) ? order_of(g.weights[small_at(p, i - at * page_size)]) : 0u;
        };
        auto key = [&](int i) { return i - lo < g.keys ? keys[i - lo] : look_up(i); };
        for (int i = threadIdx.x; i < 4 * 256; i += THREADS) (&hist[0][0])[i] = 0u;
        __syncthreads();
        // the wanted-th largest: `least`, of which `ties` are wanted
        uint32_t least = 0u;
        int ties = wanted;
        if (wanted > 0) {
            constexpr int F = 4;                          // weights of a thread in flight: their pages, then they
            for (int i0 = lo + static_cast<int>(threadIdx.x); i0 < hi; i0 += F * THREADS) {
                int p[F], t[F];
                float w[F];
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const int i = min(i0 + f * THREADS, hi - 1), at = static_cast<int>(g.by_page.div(static_cast<uint32_t>(i)));
                    p[f] = pages[at];
                    t[f] = i - at * page_size;
                }
#pragma unroll
                for (int f = 0; f < F; ++f) w[f] = in_pool(p[f]) ? g.weights[small_at(p[f], t[f])] : __uint_as_float(0x7FC00000u);
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const int i = i0 + f * THREADS;
                    if (i >= hi) break;
                    if (!in_pool(p[f])) set_status(g.status, SISO_ERR_INVALID_ARG);
                    const uint32_t x = order_of(w[f]);
                    if (i - lo < g.keys) keys[i - lo] = x;
                    atomicAdd(&hist[0][x >> 24], 1u);
                }
            }
            for (int pass = 0;; ++pass) {
                const int shift = 24 - 8 * pass;
                together();
                const uint32_t *h = hist[pass];
                if (n_ctas > 1) {
                    uint32_t *sum = sums[pass & 1];
                    if (threadIdx.x < 256) {
                        uint32_t all = 0u;
                        for (uint32_t c = 0; c < n_ctas; ++c) all += remote(&hist[pass][threadIdx.x], c);
                        sum[threadIdx.x] = all;
                    }
                    __syncthreads();
                    h = sum;
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
                uint32_t *below = hist[pass + 1];
                for (int i = lo + static_cast<int>(threadIdx.x); i < hi; i += THREADS) {
                    const uint32_t x = key(i);
                    if (x >> shift == least >> shift) atomicAdd(&below[(x >> (shift - 8)) & 255u], 1u);
                }
            }
        }
        // how many of each warp's places are heavier, and as heavy
        const int warp_each = each / WARPS, w_lo = min(hi, lo + warp * warp_each), w_hi = min(hi, w_lo + warp_each);
        uint32_t gt = 0u, eq = 0u;
        if (wanted > 0) {
            for (int i = w_lo + lane; i < w_hi; i += 32) {
                const uint32_t x = key(i);
                gt += x > least;
                eq += x == least;
            }
            gt = __reduce_add_sync(0xFFFFFFFFu, gt);
            eq = __reduce_add_sync(0xFFFFFFFFu, eq);
        }
        if (lane == 0) { warp_gt[warp] = gt; warp_eq[warp] = eq; }
        __syncthreads();
        uint32_t gt_before = 0u, eq_before = 0u;
        for (int w = 0; w < WARPS; ++w) {
            if (w == warp) { gt = gt_before; eq = eq_before; }
            gt_before += warp_gt[w];
            eq_before += warp_eq[w];
        }
        if (n_ctas > 1) {
            if (threadIdx.x == 0) { counts[0] = gt_before; counts[1] = eq_before; }
            cluster_sync();
            for (uint32_t c = 0; c < rank; ++c) { gt += remote(&counts[0], c); eq += remote(&counts[1], c); }
        }
        // their places in the list, in order
        if (wanted > 0)
            for (int i0 = w_lo; i0 < w_hi; i0 += 32) {
                const uint32_t x = i0 + lane < w_hi ? key(i0 + lane) : 0u;
                const bool there = i0 + lane < w_hi, more = there && x > least, same = there && x == least;
                const uint32_t is_gt = __ballot_sync(0xFFFFFFFFu, more), is_eq = __ballot_sync(0xFFFFFFFFu, same), below = (1u << lane) - 1u;
                const uint32_t my_gt = gt + __popc(is_gt & below), my_eq = eq + __popc(is_eq & below);
                // (the bound holds unless weights change meanwhile, as where sequences share pages)
                const uint32_t to = my_gt + min(my_eq, static_cast<uint32_t>(ties));
                if ((more || (same && my_eq < static_cast<uint32_t>(ties))) && to < static_cast<uint32_t>(wanted)) kept[to] = i0 + lane;
                gt += __popc(is_gt);
                eq += __popc(is_eq);
            }
    }
    // whether any row may be written to a place that another row is read from
    bool same_page = false;
    for (int i = threadIdx.x; i < g.out_max_pages && static_cast<long long>(i) * page_size < n_kept; i += THREADS)
        same_page = same_page || (i < g.max_pages && out_pages[i] == pages[i]);
    const bool in_place = __syncthreads_or(same_page) != 0;
    __threadfence();
    together();

    // ---- the rows move, `wave` tokens at a time
    // tokens that the CTA takes side by side: no more than leave it a thread for the small things of each of U times as many
    const int per_token = 2 * g.p.pieces, tokens_step = min(THREADS / per_token, THREADS / U), cta_wave = tokens_step * U;
    const int off = static_cast<int>(threadIdx.x) / per_token, item = static_cast<int>(threadIdx.x) - off * per_token;
    const bool is_v = item >= g.p.pieces;
    char *base = (is_v ? g.p.v : g.p.k) + layer * g.p.stride_layer + head * g.p.stride_head + (is_v ? item - g.p.pieces : item) * PIECE;
    for (int w0 = 0; w0 < n_kept; w0 += cta_wave * static_cast<int>(n_ctas)) {
        // thread i: where the i-th of the CTA's tokens comes from and goes to, and its weight and exponents
        const int t_mine = w0 + static_cast<int>(rank) * cta_wave + static_cast<int>(threadIdx.x);
        long long small_to = -1;
        float weight = 0.f;
        uint8_t ke = 0, ve = 0;
        if (static_cast<int>(threadIdx.x) < cta_wave) {
            int4 m = make_int4(-1, 0, 0, 0);
            if (t_mine < n_kept) {
                const int j = kept[t_mine];
                if (j >= t_mine && j < len) {                                     // (always, unless sequences share pages, see above)
                    const int i0 = static_cast<int>(g.by_page.div(static_cast<uint32_t>(j))), i1 = static_cast<int>(g.by_page.div(static_cast<uint32_t>(t_mine)));
                    const int p0 = pages[i0], p1 = i1 < g.out_max_pages ? out_pages[i1] : -1;
                    if (!in_pool(p0) || !in_pool(p1)) set_status(g.status, SISO_ERR_INVALID_ARG);
                    else if (p0 != p1 || j - i0 * page_size != t_mine - i1 * page_size) m = make_int4(p0, j - i0 * page_size, p1, t_mine - i1 * page_size);
                }
            }
            moves[threadIdx.x] = m;
            if (m.x >= 0) {
                const long long from = small_at(m.x, m.y);
                small_to = small_at(m.z, m.w);
                weight = g.weights[from];
                if (g.p.k_exp) { ke = g.p.k_exp[from]; ve = g.p.v_exp[from]; }
            }
        }
        __syncthreads();
        T x[U];
        if (off < tokens_step)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int4 m = moves[u * tokens_step + off];
                if (m.x >= 0) x[u] = *reinterpret_cast<const T *>(base + m.x * g.p.stride_page + m.y * g.p.stride_token);
            }
        if (in_place) together();
        if (off < tokens_step)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int4 m = moves[u * tokens_step + off];
                if (m.x >= 0) *reinterpret_cast<T *>(base + m.z * g.p.stride_page + m.w * g.p.stride_token) = x[u];
            }
        if (small_to >= 0) {
            g.weights[small_to] = weight;
            if (g.p.k_exp) { g.p.k_exp[small_to] = ke; g.p.v_exp[small_to] = ve; }
        }
        __syncthreads();                          // (`moves` is read until here)
    }
    if (n_ctas > 1) cluster_sync();               // (no CTA leaves while another reads its shared memory)
}

template <int PIECE> static siso_status_t run_evict(Kv *h, const EvictArgs &g0, int max_cand, cudaStream_t s) {
    EvictArgs g = g0;
    const long long segs = static_cast<long long>(g.p.n_layers) * g.n_seqs * g.p.n_kv_heads;
    // as many CTAs for each as keep the SMs busy, and as the list and its rows give work for
    int ctas = 1;
    while (ctas < 8 && segs * ctas < 2ll * h->sm_count) ctas *= 2;
    if (segs * ctas >= (1ll << 31)) return SISO_ERR_UNSUPPORTED;
    const int each = ((max_cand + ctas - 1) / ctas + THREADS - 1) / THREADS * THREADS;
    g.keys = std::min(KEYS, each);
    const size_t smem = static_cast<size_t>(g.keys) * 4;
    constexpr uint32_t bit = 1u << 16;
    if (!(h->attr_set & bit)) {
        SISO_CUDA(cudaFuncSetAttribute(evict_kernel<PIECE>, cudaFuncAttributeMaxDynamicSharedMemorySize, KEYS * 4));
        h->attr_set |= bit;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(segs * ctas));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SISO_CUDA(cudaLaunchKernelEx(&cfg, evict_kernel<PIECE>, g));
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
    g.items = 2 * g.p.n_kv_heads * (g.p.pieces + (g.p.k_exp ? 1 : 0));
    g.status = h->status;
    const int z = std::min(64, (g.items + kve::KEEP_THREADS - 1) / kve::KEEP_THREADS);
    const dim3 grid(static_cast<unsigned>(n_seqs), static_cast<unsigned>(g.p.n_layers), static_cast<unsigned>(z));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (piece == 16) kve::keep_path_kernel<16><<<grid, kve::KEEP_THREADS, 0, s>>>(g);
    else kve::keep_path_kernel<8><<<grid, kve::KEEP_THREADS, 0, s>>>(g);
    SISO_CUDA(cudaGetLastError());
    return SISO_OK;
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
