// Trees of drafted tokens: which nodes lie above which, and the verification of a tree against the target's probabilities.
//
// Verification.  From node 0 on, with p the target's row of the node, q the row its children were drawn from (no such rows: the children
// were certain, q = [v = x] for child x), r = p and s = 1, the children are tried in order:
//     child c with token x stands if u_c (s q(x)) < r(x);  the walk goes on from it with r = its p, s = 1
//     otherwise  r <- max(r - s q, 0),  s <- 2^-38 fp32(sum of floor(min(r, 1) 2^38))
// and where none stands the next token is drawn from r.  r / s is what is left of the target once the tried children's share is taken
// off, so the tokens are distributed as the target's whatever the drafts are (children drawn independently from q, or distinct certain
// ones).  Every product and difference is rounded to fp32 by itself and sums are whole numbers, so the result does not depend on how a
// row is split, and a chain gives what the verification of a chain gives.
//
// A row has to be read only at nodes where a child falls or the walk ends; until then the walk needs p and q at the children's tokens alone,
// which all CTAs fetch for all nodes at the start.  A cluster of CTAs shares a sequence: each warp owns one contiguous chunk of the vocabulary,
// r stays in shared memory (fp32) from the first fall at a node on, and the chunk sums go to every CTA through distributed shared memory.
// Bound by latency: a fall is a pass over the row and a cluster barrier, and the next child's turn comes after it.  Measured: 32 trees of 9 to 25 nodes over 128,256 bf16
// 31 us; one of 16 nodes over 32,000 fp32 12 to 14 us.
#include "kv.cuh"

namespace siso {
namespace tree {

// ---- ancestors -----------------------------------------------------------------------------------------------------------
// A CTA per sequence, a thread per node.  Parents come before their children, so a node's walk upwards meets the words of its
// row from the last to the first: one word is built in a register at a time.  Bound by latency: a step is one load from shared memory.
constexpr int MASK_THREADS = 128, MASK_NODES = 4096;          // nodes whose parents are kept in shared memory
__global__ void __launch_bounds__(MASK_THREADS)
tree_mask_kernel(const int32_t *__restrict__ parents, const int32_t *__restrict__ cu_q, int n_tokens, int words, uint32_t *__restrict__ mask,
                 int32_t *__restrict__ depth) {
    __shared__ int32_t near[MASK_NODES];
    wait_for_earlier();
    dependents_may_start();
    const int lo = min(max(cu_q[blockIdx.x], 0), n_tokens), n = max(0, min(cu_q[blockIdx.x + 1], n_tokens) - lo);
    for (int i = threadIdx.x; i < min(n, MASK_NODES); i += MASK_THREADS) near[i] = parents[lo + i];
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += MASK_THREADS) {
        uint32_t *row = mask + static_cast<long long>(lo + i) * words;
        uint32_t bits = 0u;
        int word = words - 1, above = 0;
        for (int a = i;;) {
            for (; word > (a >> 5); --word) {
                row[word] = bits;
                bits = 0u;
            }
            if (word == (a >> 5)) bits |= 1u << (a & 31);
            const int up = a < MASK_NODES ? near[a] : parents[lo + a];
            if (up < 0 || up >= a) break;
            a = up;
            ++above;
        }
        for (; word >= 0; --word) {
            row[word] = bits;
            bits = 0u;
        }
        if (depth) depth[lo + i] = above;
    }
}

// ---- verification --------------------------------------------------------------------------------------------------------
constexpr int THREADS = 512, WARPS = THREADS / 32, SPLIT = 8, CHUNKS = SPLIT * WARPS;
constexpr int NODES = 512;                        // nodes whose numbers are kept in shared memory
constexpr int MAX_VOCAB = 1 << 18;                // a CTA's part of r is 128 KB of its shared memory then; eight CTAs could hold over 400,000 entries, but nothing has asked for more

struct Args {
    const void *target, *draft;                   // [n_tokens, vocab]
    const int32_t *tokens, *parents, *cu_q;
    const float *u_accept, *u_sample;
    int32_t *out, *accepted, *path;
    int n_tokens, vocab, max_path, chunk;         // chunk: entries of a warp, a multiple of 8
};
template <typename T> __device__ __forceinline__ float value(const T *p) {
    if constexpr (sizeof(T) == 2) return __bfloat162float(*p); else return *p;
}
// 38-bit weight; NaN and negative values weigh nothing
__device__ __forceinline__ unsigned long long weight(float r) { return __float2ull_rz(__saturatef(r) * 274877906944.f); }
// Sum of such weights of a few entries without 64-bit conversions: an entry times 2^22 is split at its binary point by an addition that rounds down (the whole number
// then stands in the low bits), what is left times 2^16 is rounded down the same way.  Up to 256 entries
struct Weights {
    uint32_t high = 0u, low = 0u, n = 0u;
    __device__ __forceinline__ void add(float r) {
        const float y = __saturatef(r), t = __fmaf_rd(y, 4194304.f, 8388608.f), u = __fmaf_rd(fmaf(y, 4194304.f, 8388608.f - t), 65536.f, 8388608.f);
        high += __float_as_uint(t);
        low += __float_as_uint(u);
        ++n;
    }
    __device__ __forceinline__ unsigned long long sum() const {
        return (static_cast<unsigned long long>(high - n * 0x4B000000u) << 16) + (low - n * 0x4B000000u);
    }
};
__device__ __forceinline__ float left_of(float r, float s, float q) { return fmaxf(__fsub_rn(r, __fmul_rn(s, q)), 0.f); }
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// The same word of shared memory in CTA `rank` of the cluster is written
__device__ __forceinline__ void put_in(const float *p, uint32_t rank, float x) {
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(x) : "memory");
}
__device__ __forceinline__ unsigned long long warp_sum(unsigned long long x) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
__device__ __forceinline__ unsigned long long warp_scan(unsigned long long x, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}
// 8 consecutive entries as they lie in memory; WIDE: from a 16-byte boundary, all of them there
template <typename T, bool WIDE> struct Eight {
    static constexpr int N = WIDE && sizeof(T) == 2 ? 4 : 8;
    uint32_t w[N];
    __device__ __forceinline__ void load(const T *p, int there) {
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const uint4 r = reinterpret_cast<const uint4 *>(p)[i / 4];
                w[i] = r.x; w[i + 1] = r.y; w[i + 2] = r.z; w[i + 3] = r.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < there ? __float_as_uint(value(p + i)) : 0u;
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (N == 8) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
};

template <typename T, bool WIDE>
__global__ void __cluster_dims__(SPLIT, 1, 1) __launch_bounds__(THREADS, 2)
verify_tree_kernel(Args g) {
    extern __shared__ __align__(16) float r[];                       // this CTA's part of r, [WARPS * chunk]
    __shared__ unsigned long long sums[2][CHUNKS], scan[WARPS];
    __shared__ int32_t parent[NODES], token[NODES];
    __shared__ float p_at[NODES], q_at[NODES], u_at[NODES];          // r and q at a node's token, in its parent's rows; its u_accept
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    wait_for_earlier();
    dependents_may_start();
    // said here, waited for below: a CTA's shared memory may be written by others only once it is known to have started
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int b = blockIdx.x / SPLIT;
    const int lo = min(max(g.cu_q[b], 0), g.n_tokens), n_nodes = max(0, min(g.cu_q[b + 1], g.n_tokens) - lo);
    const T *target = static_cast<const T *>(g.target) + static_cast<long long>(lo) * g.vocab;
    const T *draft = g.draft ? static_cast<const T *>(g.draft) + static_cast<long long>(lo) * g.vocab : nullptr;

    auto parent_of = [&](int i) { const int up = i < NODES ? parent[i] : g.parents[lo + i]; return up < i ? up : -1; };
    auto token_of = [&](int i) { return i < NODES ? token[i] : g.tokens[lo + i]; };
    auto in_vocab = [&](int x) { return x >= 0 && x < g.vocab; };
    for (int i = threadIdx.x; i < min(n_nodes, NODES); i += THREADS) {
        parent[i] = g.parents[lo + i];
        token[i] = g.tokens[lo + i];
        u_at[i] = g.u_accept[lo + i];
    }
    // each CTA fetches p and q of every eighth node and gives them to all: rows are far apart, and what their addresses cost to translate is paid once (32 trees of
    // 9 to 25 nodes: 31 us and 33 us with every CTA fetching all)
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    for (int i = static_cast<int>(rank) + SPLIT * static_cast<int>(threadIdx.x); i < min(n_nodes, NODES); i += SPLIT * THREADS) {
        const int up = g.parents[lo + i], x = g.tokens[lo + i];
        float p = 0.f, q = 1.f;
        if (up >= 0 && up < i && in_vocab(x)) {
            const long long at = static_cast<long long>(up) * g.vocab + x;
            p = value(target + at);
            if (draft) q = value(draft + at);
        }
        for (uint32_t c = 0; c < SPLIT; ++c) {
            put_in(p_at + i, c, p);
            put_in(q_at + i, c, q);
        }
    }
    cluster_sync();

    const int first = (static_cast<int>(rank) * WARPS + warp) * g.chunk;                 // this warp's chunk
    const int lo_v = min(g.vocab, first), hi_v = min(g.vocab, first + g.chunk);
    float *mine = r + warp * g.chunk - lo_v;
    const int cta_lo = static_cast<int>(rank) * WARPS * g.chunk;
    int passes = 0;
    // Goes over the row of node `at`: r from shared memory (again) or the target's row, less s q or without entry `without`.  Leaves the chunk sums
    // at sums[(passes - 1) & 1] and returns their sum
    auto pass = [&](int at, bool again, bool less, float s, int without) {
        const T *p = target + static_cast<long long>(at) * g.vocab, *q = draft + static_cast<long long>(at) * g.vocab;
        Weights weights;
        constexpr int F = WIDE && sizeof(T) == 2 ? 4 : 2;      // eights of a lane in flight: with the rows in DRAM a trip takes over a microsecond
        for (int v0 = lo_v + lane * 8; v0 < hi_v; v0 += F * 256) {
            Eight<T, WIDE> x[F], y[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int v = v0 + f * 256;
                if (!again && v < hi_v) x[f].load(p + v, hi_v - v);
                if (less && v < hi_v) y[f].load(q + v, hi_v - v);
            }
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int v = v0 + f * 256;
                if (v >= hi_v) continue;
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    if (again) *reinterpret_cast<float4 *>(z + i) = *reinterpret_cast<const float4 *>(mine + v + i);
                    else { z[i] = x[f].get(i); z[i + 1] = x[f].get(i + 1); z[i + 2] = x[f].get(i + 2); z[i + 3] = x[f].get(i + 3); }
                }
                if (less) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = left_of(z[i], s, y[f].get(i));
                }
                if (without >= v && without < v + 8) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (v + i == without) z[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) weights.add(z[i]);
#pragma unroll
                for (int i = 0; i < 8; i += 4) *reinterpret_cast<float4 *>(mine + v + i) = *reinterpret_cast<const float4 *>(z + i);
            }
        }
        unsigned long long sum = weights.sum();
        sum = warp_sum(sum);
        unsigned long long *to = sums[passes & 1];
        if (lane < SPLIT) {
            const uint32_t here = static_cast<uint32_t>(__cvta_generic_to_shared(&to[static_cast<int>(rank) * WARPS + warp]));
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(lane));
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there), "l"(sum) : "memory");
        }
        // (two sets of sums: a CTA writes a set again only after a barrier that all reach once they have read it)
        cluster_sync();
        unsigned long long all = 0ull;
        for (int c = lane; c < CHUNKS; c += 32) all += to[c];
        ++passes;
        return warp_sum(all);
    };

    // ---- the walk: every warp of every CTA makes it, with the same numbers
    int at = 0, tried = 0, n = 0;
    float s = 1.f;
    bool have = false, stale = false;             // r is in shared memory; the chunk sums are those before entries were taken out
    unsigned long long total = 0ull;
    while (n_nodes > 0) {
        int child = -1;
        if (n < g.max_path)
            for (int i0 = tried + 1; i0 < n_nodes && child < 0; i0 += 32) {
                const uint32_t is = __ballot_sync(0xFFFFFFFFu, i0 + lane < n_nodes && parent_of(i0 + lane) == at);
                if (is) child = i0 + __ffs(is) - 1;
            }
        if (child < 0) break;
        tried = child;
        const int x = token_of(child);
        const bool real = in_vocab(x);
        float rx, qx, u;
        if (child < NODES) { rx = p_at[child]; qx = q_at[child]; u = u_at[child]; }
        else {                                    // r at its token is with the CTA that owns it, or still in the target's row
            u = g.u_accept[lo + child];
            const long long place = static_cast<long long>(at) * g.vocab + (real ? x : 0);
            qx = draft && real ? value(draft + place) : 1.f;
            rx = real ? value(target + place) : 0.f;
            if (have && real) {
                const uint32_t here = static_cast<uint32_t>(__cvta_generic_to_shared(r + x % (WARPS * g.chunk)));
                uint32_t there;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(x / (WARPS * g.chunk)));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(rx) : "r"(there) : "memory");
                // nobody writes r again before all have read
                cluster_sync();
            }
        }
        if (real && __fmul_rn(u, __fmul_rn(s, qx)) < rx) {
            if (rank == 0 && threadIdx.x == 0) {
                g.out[static_cast<long long>(b) * (g.max_path + 1) + n] = x;
                if (g.path) g.path[static_cast<long long>(b) * g.max_path + n] = child;
            }
            at = child;
            ++n;
            s = 1.f;
            have = stale = false;
            continue;
        }
        // the child falls: what is left at the tokens of its sisters, and of the row
        __syncthreads();                           // (all have looked at p_at)
        for (int i = child + 1 + threadIdx.x; i < min(n_nodes, NODES); i += THREADS)
            if (parent_of(i) == at) p_at[i] = draft ? left_of(p_at[i], s, q_at[i]) : real && token[i] == x ? 0.f : p_at[i];
        if (draft || !have) {
            total = pass(at, have, draft != nullptr, s, draft ? -1 : x);
            have = true;
        } else if (real) {                         // one entry less
            if (rx > 0.f) total -= weight(rx);
            if (x >= cta_lo && x < cta_lo + WARPS * g.chunk && threadIdx.x == 0) r[x - cta_lo] = 0.f;
            stale = true;
            if (n_nodes > NODES) cluster_sync();       // (another CTA may ask for the entry)
        }
        s = __fmul_rn(__ull2float_rn(total), 3.637978807091713e-12f);          // 2^-38
        __syncthreads();
    }

    // ---- the next token is drawn from r
    if (n_nodes > 0) {
        if (!have || stale) total = pass(at, have, false, 0.f, -1);
        if (total == 0ull) total = pass(at, false, false, 0.f, -1);
    }
    if (rank == 0) {
        int32_t *out = g.out + static_cast<long long>(b) * (g.max_path + 1);
        for (int t = n + threadIdx.x; t <= g.max_path; t += THREADS) {
            if (t > n || total == 0ull) out[t] = -1;
            if (g.path && t < g.max_path) g.path[static_cast<long long>(b) * g.max_path + t] = -1;
        }
        if (threadIdx.x == 0) g.accepted[b] = n;
    }
    if (total == 0ull) return;

    // the chunk with the crossing: the first whose running sum exceeds floor(z W / 2^24)
    const unsigned long long *chunk_sums = sums[(passes - 1) & 1];
    const unsigned long long z = static_cast<unsigned long long>(fminf(fmaxf(g.u_sample[b], 0.f) * 16777216.f, 16777215.f));
    const unsigned long long cross = (__umul64hi(z, total) << 40) | ((z * total) >> 24);
    unsigned long long before = 0ull;
    int c_at = -1;
    for (int c0 = 0; c0 < CHUNKS && c_at < 0; c0 += 32) {
        const unsigned long long part = chunk_sums[c0 + lane], upto = before + warp_scan(part, lane);
        const uint32_t over = __ballot_sync(0xFFFFFFFFu, upto > cross);
        if (over) {
            const int f = __ffs(over) - 1;
            c_at = c0 + f;
            before = __shfl_sync(0xFFFFFFFFu, upto - part, f);
        } else {
            before = __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    }
    if (c_at < 0 || c_at / WARPS != static_cast<int>(rank)) return;
    // the entry: consecutive ones per thread, a scan over the CTA
    __syncthreads();
    const int c_lo = c_at * g.chunk, c_hi = min(g.vocab, c_lo + g.chunk), each = (g.chunk + THREADS - 1) / THREADS;
    const int v0 = min(c_hi, c_lo + static_cast<int>(threadIdx.x) * each), v1 = min(c_hi, v0 + each);
    unsigned long long sum = 0ull;
    for (int v = v0; v < v1; ++v) sum += weight(r[v - cta_lo]);
    const unsigned long long upto = warp_scan(sum, lane);
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    unsigned long long start = before + upto - sum;
    for (int w = 0; w < warp; ++w) start += scan[w];
    if (start <= cross && start + sum > cross) {          // exactly one thread
        int v = v0;
        for (; v < v1 - 1; ++v) {
            start += weight(r[v - cta_lo]);
            if (start > cross) break;
        }
        g.out[static_cast<long long>(b) * (g.max_path + 1) + n] = v;
    }
}

template <typename T, bool WIDE> static siso_status_t run(const Args &g, int n_seqs, cudaStream_t s) {
    constexpr int MOST = MAX_VOCAB / SPLIT * static_cast<int>(sizeof(float));
    static_assert(MAX_VOCAB % (CHUNKS * 8) == 0, "a CTA's part of the largest vocabulary is no larger than its share");
    const int smem = WARPS * g.chunk * static_cast<int>(sizeof(float));
    // asked for at every call, as which device the function has it on is not known here; always the most that any call takes, or one thread's call would
    // take it from another's between its asking and its launch
    if (smem > 24 * 1024) SISO_CUDA(cudaFuncSetAttribute(verify_tree_kernel<T, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST));
    return launch_early(verify_tree_kernel<T, WIDE>, dim3(static_cast<unsigned>(n_seqs) * SPLIT), THREADS, static_cast<size_t>(smem), s, g);
}

}  // namespace tree
}  // namespace siso

using namespace siso;

extern "C" siso_status_t siso_tree_mask(const int32_t *d_parents, const int32_t *d_cu_q, int64_t n_tokens, int32_t n_seqs, int32_t words,
                                        uint32_t *d_mask, int32_t *d_depth, void *stream) {
    if (n_tokens < 0 || n_seqs < 0 || words < 1) return SISO_ERR_INVALID_ARG;
    if (n_tokens == 0 || n_seqs == 0) return SISO_OK;
    if (!d_parents || !d_cu_q || !d_mask) return SISO_ERR_INVALID_ARG;
    if (n_tokens >= (1ll << 31)) return SISO_ERR_UNSUPPORTED;
    return launch_early(tree::tree_mask_kernel, dim3(static_cast<unsigned>(n_seqs)), tree::MASK_THREADS, 0, static_cast<cudaStream_t>(stream), d_parents, d_cu_q,
                        static_cast<int>(n_tokens), words, d_mask, d_depth);
}

extern "C" siso_status_t siso_verify_tree(const void *d_target, const void *d_draft, int32_t dtype, int64_t n_tokens, int32_t n_seqs, int32_t vocab,
                                          const int32_t *d_tokens, const int32_t *d_parents, const int32_t *d_cu_q, int32_t max_path,
                                          const float *d_u_accept, const float *d_u_sample, int32_t *d_out, int32_t *d_accepted,
                                          int32_t *d_path, void *stream) {
    if (dtype != SISO_F32 && dtype != SISO_BF16) return SISO_ERR_INVALID_ARG;
    if (n_tokens < 0 || n_seqs < 0 || max_path < 0 || vocab < 1) return SISO_ERR_INVALID_ARG;
    if (n_seqs == 0) return SISO_OK;
    if (!d_cu_q || !d_u_sample || !d_out || !d_accepted || (n_tokens > 0 && (!d_target || !d_tokens || !d_parents || !d_u_accept)))
        return SISO_ERR_INVALID_ARG;
    if (vocab > tree::MAX_VOCAB || n_tokens >= (1ll << 31) || n_seqs > (1 << 27) || max_path == 0x7FFFFFFF) return SISO_ERR_UNSUPPORTED;
    const int chunk = ((vocab + tree::CHUNKS - 1) / tree::CHUNKS + 7) & ~7;
    const tree::Args g{d_target, d_draft, d_tokens, d_parents, d_cu_q, d_u_accept, d_u_sample, d_out, d_accepted, d_path,
                       static_cast<int>(n_tokens), vocab, max_path, chunk};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // 8 entries at a time where every row starts on a boundary of 16 bytes and is made of whole eights
    const bool wide = vocab % 8 == 0 && ((reinterpret_cast<uintptr_t>(d_target) | reinterpret_cast<uintptr_t>(d_draft)) & 15u) == 0;
    if (dtype == SISO_F32) return wide ? tree::run<float, true>(g, n_seqs, s) : tree::run<float, false>(g, n_seqs, s);
    return wide ? tree::run<__nv_bfloat16, true>(g, n_seqs, s) : tree::run<__nv_bfloat16, false>(g, n_seqs, s);
}
