// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// Draft t of a sequence is token x_t.  p_t is the target's row at t, q_t the row the draft was drawn from (no draft rows: x_t
// was certain, q_t = [v = x_t]).  With u_t uniform in [0, 1):
//     draft t stands if u_t q_t(x_t) < p_t(x_t);   n = the first that does not, or the number of drafts
//     the next token is drawn from r = max(p_n - q_n, 0), or from p_n where every draft stands
// which leaves the tokens distributed as the target's.  The draw inverts the distribution in whole numbers:
//     w_v = floor(min(r_v, 1) 2^38),  W = sum of all w,  z = floor(u 2^24),  token = smallest v with 2^24 (w_0 + ... + w_v) > z W
// Whole numbers add up to the same sum in any order, so the token does not depend on how the row is split, and a row of
// 2^24 entries of at most 2^38 stays inside 64 bits.  Truncation moves a probability by at most 2^-38, less than an fp32 sum over
// a vocabulary would.  Where the residual is empty (q_n >= p_n everywhere) the draw is from p_n; where that is empty too
// the token is -1.
//
// Only row n of p and of q has to be read, so the call is bound by latency for one sequence and by HBM for many.  A cluster of
// up to 8 CTAs shares a sequence: each warp sums the weights of one contiguous chunk, the chunk sums go to every CTA of the
// cluster through distributed shared memory, and the CTA that owns the chunk with the crossing looks at it again (it comes
// from L2) with a few consecutive entries per thread.  One launch, no scratch memory.
// Measured with rows in HBM: 64 x 128256 fp32 (66 MB) 14.4 us, 4.6 TB/s; 192 x 50257 bf16 (39 MB, rows not aligned) 16.5 us, 2.3 TB/s; one
// sequence of 32000 fp32 4.4 us, most of it the launch and three round trips to memory (which drafts stand, the row, the crossing).
#include "common.cuh"

namespace siso {
namespace ver {

struct Args {
    const void *target, *draft;          // [n_seqs, n_max + 1, vocab], [n_seqs, n_max, vocab] or NULL
    const int32_t *tokens, *n_drafts;    // [n_seqs, n_max], [n_seqs] or NULL
    const float *u_accept, *u_sample;    // [n_seqs, n_max], [n_seqs]
    int32_t *out, *accepted;             // [n_seqs, n_max + 1], [n_seqs]
    int n_max, vocab;
};

template <typename T> __device__ __forceinline__ float value(const T *p) {
    if constexpr (sizeof(T) == 2) return __bfloat162float(*p); else return *p;
}
// Loads that stay where they are written: left to itself the compiler takes them one by one to save registers
__device__ __forceinline__ float load_now(const float *p) {
    float x;
    asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(x) : "l"(p));
    return x;
}
__device__ __forceinline__ float load_now(const __nv_bfloat16 *p) {
    uint16_t x;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(x) : "l"(p));
    return __uint_as_float(static_cast<uint32_t>(x) << 16);
}
// 38-bit weight of a probability or a difference of two; NaN and negative values weigh nothing
__device__ __forceinline__ unsigned long long weight(float r) { return __float2ull_rz(__saturatef(r) * 274877906944.f); }
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

// r_v of the row that the next token is drawn from: without = the entry to leave out (certain draft), q = NULL: nothing taken off
template <typename T> struct Residual {
    const T *p, *q;
    int without;
    __device__ __forceinline__ float at(int v) const {
        const float a = value(p + v);
        if (q) return a - value(q + v);
        return v == without ? 0.f : a;
    }
};

// 16 bytes of entries at once
template <typename T, int W> struct Some {
    uint4 r;
    __device__ __forceinline__ void load(const T *p) {
        asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    }
    __device__ __forceinline__ void clear() { r = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ float get(int i) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
        if constexpr (W == 4) return __uint_as_float(w[i]);
        return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
};
// This lane's weights of the entries [lo, hi), whose ends are whole pieces of W.  U pieces of each row are in flight: with the rows in DRAM a
// round of loads takes over a microsecond, so rounds are what a call's time is made of
template <typename T, int W, int U, bool Q>
__device__ __forceinline__ unsigned long long chunk_sum(const Residual<T> &r, int lo, int hi, int lane) {
    unsigned long long sum = 0ull;
    if constexpr (W == 1) {
        int v0 = lo;                   // (entry by entry, tests of the end cost more than they are worth: 192 x 50257 bf16 31 us and 15.6 us)
        for (; v0 + 32 * U <= hi; v0 += 32 * U) {
            float a[U], b[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                a[i] = load_now(r.p + v0 + 32 * i + lane);
                b[i] = Q ? load_now(r.q + v0 + 32 * i + lane) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < U; ++i) sum += !Q && v0 + 32 * i + lane == r.without ? 0ull : weight(a[i] - b[i]);
        }
        for (v0 += lane; v0 < hi; v0 += 32 * U) {
            float x[U];
#pragma unroll
            for (int i = 0; i < U; ++i) x[i] = v0 + 32 * i < hi ? r.at(v0 + 32 * i) : 0.f;
#pragma unroll
            for (int i = 0; i < U; ++i) sum += weight(x[i]);
        }
    } else {
        for (int v0 = lo + lane * W; v0 < hi; v0 += 32 * W * U) {
            Some<T, W> a[U], b[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int v = v0 + 32 * W * i;
                a[i].clear();
                b[i].clear();
                if (v < hi) {
                    a[i].load(r.p + v);
                    if (Q) b[i].load(r.q + v);
                }
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int w = 0; w < W; ++w)
                    sum += Q ? weight(a[i].get(w) - b[i].get(w)) : v0 + 32 * W * i + w == r.without ? 0ull : weight(a[i].get(w));
        }
    }
    return sum;
}

template <typename T, int W, int THREADS, int SPLIT>
__global__ void __cluster_dims__(SPLIT, 1, 1) __launch_bounds__(THREADS)
verify_kernel(Args g) {
    constexpr int WARPS = THREADS / 32;
    __shared__ unsigned long long sums[2][SPLIT * WARPS];
    __shared__ unsigned long long scan[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t rank;
    constexpr int split = SPLIT;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    // said here, waited for below: a CTA's shared memory may be written by others only once it is known to have started
    if constexpr (SPLIT > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const long long b = blockIdx.x / split;

    // ---- which drafts stand: every warp finds it for itself
    const int limit = g.n_drafts ? min(max(g.n_drafts[b], 0), g.n_max) : g.n_max;
    const T *target = static_cast<const T *>(g.target) + b * (g.n_max + 1) * static_cast<long long>(g.vocab);
    const T *draft = g.draft ? static_cast<const T *>(g.draft) + b * g.n_max * static_cast<long long>(g.vocab) : nullptr;
    int n = limit;
    for (int t0 = 0; t0 < limit; t0 += 32) {
        const int t = t0 + lane;
        bool stands = true;
        if (t < limit) {
            const int x = g.tokens[b * g.n_max + t];
            stands = false;
            if (x >= 0 && x < g.vocab) {
                const long long at = static_cast<long long>(t) * g.vocab + x;
                const float q = draft ? value(draft + at) : 1.f;
                stands = g.u_accept[b * g.n_max + t] * q < value(target + at);
            }
        }
        const uint32_t fails = __ballot_sync(0xFFFFFFFFu, !stands);
        if (fails) { n = t0 + __ffs(fails) - 1; break; }
    }
    Residual<T> r;
    r.p = target + static_cast<long long>(n) * g.vocab;
    r.q = n < limit && draft ? draft + static_cast<long long>(n) * g.vocab : nullptr;
    r.without = n < limit && !draft ? g.tokens[b * g.n_max + n] : -1;

    // ---- sums of the chunks, one per warp of the cluster
    const int chunks = split * WARPS;
    const int chunk = ((g.vocab + chunks - 1) / chunks + 7) & ~7;      // whole pieces of 16 bytes
    const int me = static_cast<int>(rank) * WARPS + warp;
    unsigned long long total = 0ull;
    int pass = 0;
    for (; pass < 2; ++pass) {
        const int lo = min(g.vocab, me * chunk), hi = min(g.vocab, lo + chunk);
        constexpr int U = W == 1 ? 16 : 4;       // (192 x 50257 bf16, entry by entry: 8 20.3 us, 16 15.1 us; 64 x 128256 fp32: 2 14.5 us, 4 13.5 us)
        unsigned long long sum = r.q ? chunk_sum<T, W, U, true>(r, lo, hi, lane) : chunk_sum<T, W, U, false>(r, lo, hi, lane);
        sum = warp_sum(sum);
        if (SPLIT > 1 && pass == 0) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (lane < split) {
            const uint32_t here = static_cast<uint32_t>(__cvta_generic_to_shared(&sums[pass][me]));
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(lane));
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there), "l"(sum) : "memory");
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        total = 0ull;
        for (int c = lane; c < chunks; c += 32) total += sums[pass][c];
        total = warp_sum(total);
        if (total != 0ull) break;
        r.q = nullptr;                    // nothing to draw from: from the target's row itself
        r.without = -1;
    }

    if (rank == 0) {
        for (int t = threadIdx.x; t <= g.n_max; t += THREADS)
            if (t != n || total == 0ull) g.out[b * (g.n_max + 1) + t] = t < n ? g.tokens[b * g.n_max + t] : -1;
        if (threadIdx.x == 0) g.accepted[b] = n;
    }
    if (total == 0ull) return;

    // ---- the chunk with the crossing: first whose running sum exceeds floor(z W / 2^24)
    const float u = g.u_sample[b];
    const unsigned long long z = static_cast<unsigned long long>(fminf(fmaxf(u, 0.f) * 16777216.f, 16777215.f));
    const unsigned long long cross = (__umul64hi(z, total) << 40) | ((z * total) >> 24);
    unsigned long long before = 0ull;
    int at = -1;
    for (int c0 = 0; c0 < chunks && at < 0; c0 += 32) {
        const unsigned long long mine = c0 + lane < chunks ? sums[pass][c0 + lane] : 0ull;
        const unsigned long long upto = before + warp_scan(mine, lane);
        const uint32_t over = __ballot_sync(0xFFFFFFFFu, upto > cross);
        if (over) {
            const int f = __ffs(over) - 1;
            at = c0 + f;
            before = __shfl_sync(0xFFFFFFFFu, upto - mine, f);
        } else {
            before = __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    }
    if (at < 0 || at / WARPS != static_cast<int>(rank)) return;
    // ---- the entry: consecutive ones per thread, a scan over the CTA
    const int lo = at * chunk, hi = min(g.vocab, lo + chunk);
    const int each = (chunk + THREADS - 1) / THREADS;
    const int v0 = lo + static_cast<int>(threadIdx.x) * each, v1 = min(hi, v0 + each);
    unsigned long long sum = 0ull;
    for (int v = v0; v < v1; ++v) sum += weight(r.at(v));
    const unsigned long long upto = warp_scan(sum, lane);
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    unsigned long long start = before + upto - sum;
    for (int w = 0; w < warp; ++w) start += scan[w];
    if (start <= cross && start + sum > cross) {          // exactly one thread
        int v = v0;
        for (; v < v1 - 1; ++v) {
            start += weight(r.at(v));
            if (start > cross) break;
        }
        g.out[b * (g.n_max + 1) + n] = v;
    }
}

// (the cluster's size is the kernel's own: 192 x 50257 bf16 13.8 us with a size given at launch, 12.8 us so)
template <typename T, int W, int THREADS, int SPLIT> static siso_status_t launch(const Args &g, int64_t n_seqs, cudaStream_t s) {
    verify_kernel<T, W, THREADS, SPLIT><<<static_cast<unsigned>(n_seqs * SPLIT), THREADS, 0, s>>>(g);
    SISO_CUDA(cudaGetLastError());
    return SISO_OK;
}
template <typename T, int W> static siso_status_t run(const Args &g, int64_t n_seqs, cudaStream_t s) {
    // A sequence is shared by as many CTAs as give each of the 148 SMs a few, small enough that all of them run at once (64 x 128256
    // fp32: 256 threads 13.4 us, 512 threads 17.3 us; 192 x 50257 bf16: four CTAs 13.6 us, two 15.1 us; 512 x 32000 fp32: two 32.8 us,
    // one 34.8 us; each with part of the rows in L2).  Few sequences with long rows get larger CTAs, fewer rounds of loads (4 x 128256 fp32: 512 threads 6.5 us, 256
    // threads 7.7 us; 1 x 32000: 4.2 us and 3.8 us)
    if (n_seqs <= 16 && g.vocab >= 65536) return launch<T, W, 512, 8>(g, n_seqs, s);
    if (n_seqs <= 64) return launch<T, W, 256, 8>(g, n_seqs, s);
    if (n_seqs <= 256) return launch<T, W, 256, 4>(g, n_seqs, s);
    if (n_seqs <= 512) return launch<T, W, 256, 2>(g, n_seqs, s);
    return launch<T, W, 256, 1>(g, n_seqs, s);
}

}  // namespace ver
}  // namespace siso

using namespace siso;

extern "C" siso_status_t siso_verify_drafts(const void *d_target, const void *d_draft, int32_t dtype, int64_t n_seqs, int32_t n_max,
                                            int32_t vocab, const int32_t *d_tokens, const int32_t *d_n_drafts, const float *d_u_accept,
                                            const float *d_u_sample, int32_t *d_out, int32_t *d_accepted, void *stream) {
    if (dtype != SISO_F32 && dtype != SISO_BF16) return SISO_ERR_INVALID_ARG;
    if (n_seqs < 0 || n_max < 0 || vocab < 1) return SISO_ERR_INVALID_ARG;
    if (n_seqs == 0) return SISO_OK;
    if (!d_target || !d_u_sample || !d_out || !d_accepted || (n_max > 0 && (!d_tokens || !d_u_accept))) return SISO_ERR_INVALID_ARG;
    if (vocab > (1 << 24) || n_seqs > (1ll << 27)) return SISO_ERR_UNSUPPORTED;
    const ver::Args g{d_target, n_max > 0 ? d_draft : nullptr, d_tokens, d_n_drafts, d_u_accept, d_u_sample, d_out, d_accepted, n_max, vocab};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // 16 bytes at a time where every row starts on a boundary of 16 bytes
    const bool wide = vocab % (dtype == SISO_F32 ? 4 : 8) == 0 && ((reinterpret_cast<uintptr_t>(d_target) | reinterpret_cast<uintptr_t>(g.draft)) & 15u) == 0;
    if (dtype == SISO_F32) return wide ? ver::run<float, 4>(g, n_seqs, s) : ver::run<float, 1>(g, n_seqs, s);
    return wide ? ver::run<__nv_bfloat16, 8>(g, n_seqs, s) : ver::run<__nv_bfloat16, 1>(g, n_seqs, s);
}
