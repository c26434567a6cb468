// Attention of a chunk of new tokens over the paged key/value cache.
//
// Token i of sequence b (q_len new tokens, already in the cache, kv_len tokens in all) stands at p = kv_len - q_len + i and
// sees the tokens j in [0, kv_len) with j <= p (causal) and j > p - window (window > 0):
//     s_j = scale q.k_j,  m = max s,  l = sum exp(s_j - m),  out = sum exp(s_j - m) v_j / l,  lse = m + ln l
// A row that sees nothing gives out = 0 and lse = -infinity.
//
// One warp owns one (token, head) row, a lane owns head_dim / 32 of its dimensions, and keys are taken one by one with the
// running maximum and sum.
#include "kv.cuh"

namespace siso {
namespace kva {

struct Args {
    KvView kv;
    siso_attention_t a;
};

template <int KIND, int D>
__global__ void __launch_bounds__(128)
attention_rows_kernel(Args g, int *status) {
    constexpr int N = D / 32;
    const int lane = threadIdx.x & 31;
    const long long row = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    const siso_attention_t &a = g.a;
    if (row >= a.n_tokens * a.n_heads) return;
    const int tok = static_cast<int>(row / a.n_heads), head = static_cast<int>(row % a.n_heads);
    int b = 0;
    while (b < a.n_seqs && !(tok >= a.d_cu_q[b] && tok < a.d_cu_q[b + 1])) ++b;
    if (b == a.n_seqs) return;
    const int kv_head = head / (a.n_heads / g.kv.n_kv_heads);
    const long long capacity = static_cast<long long>(a.max_pages) * g.kv.page_size;
    const int len = static_cast<int>(min(static_cast<long long>(max(a.d_kv_len[b], 0)), capacity));
    const int p = len - (a.d_cu_q[b + 1] - a.d_cu_q[b]) + tok - a.d_cu_q[b];
    const int hi = (a.flags & SISO_ATTN_CAUSAL) ? min(len, p + 1) : len;
    const int lo = a.window > 0 ? max(0, p - a.window + 1) : 0;
    float q[N], o[N], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        q[i] = __bfloat162float(static_cast<const __nv_bfloat16 *>(a.d_q)[tok * a.q_stride_token + head * a.q_stride_head + lane * N + i]) * a.scale;
        o[i] = 0.f;
    }
    for (int j = lo; j < hi; ++j) {
        const int page = a.d_pages[b * a.pages_stride + j / g.kv.page_size], t = j % g.kv.page_size;
        if (page < 0 || page >= g.kv.n_pages) {
            if (lane == 0) set_status(status, SISO_ERR_INVALID_ARG);
            continue;
        }
        const long long at = page * g.kv.stride_page + t * g.kv.stride_token + kv_head * g.kv.stride_head + lane * N;
        float k[N], v[N];
        if constexpr (KIND == SISO_BF16) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                k[i] = __bfloat162float(static_cast<const __nv_bfloat16 *>(g.kv.k)[at + i]);
                v[i] = __bfloat162float(static_cast<const __nv_bfloat16 *>(g.kv.v)[at + i]);
            }
        } else {
            const long long ex = (static_cast<long long>(page) * g.kv.n_kv_heads + kv_head) * g.kv.page_size + t;
            const float sk = kv_scale(g.kv.k_exp[ex]), sv = kv_scale(g.kv.v_exp[ex]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                k[i] = kv_code<KIND>(static_cast<const uint8_t *>(g.kv.k)[at + i], sk);
                v[i] = kv_code<KIND>(static_cast<const uint8_t *>(g.kv.v)[at + i], sv);
            }
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) s += q[i] * k[i];
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, x);
        const float m2 = fmaxf(m, s), c = __expf(m - m2), w = __expf(s - m2);
        l = l * c + w;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = o[i] * c + w * v[i];
        m = m2;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
        static_cast<__nv_bfloat16 *>(a.d_out)[tok * a.out_stride_token + head * a.out_stride_head + lane * N + i] = __float2bfloat16_rn(o[i] * inv);
    if (a.d_lse && lane == 0) a.d_lse[static_cast<long long>(tok) * a.n_heads + head] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace kva

siso_status_t launch_kv_attention(Kv *h, const siso_attention_t *a, cudaStream_t s) {
    kva::Args g{kv_view(h, a->layer), *a};
    const long long rows = a->n_tokens * a->n_heads;
    const unsigned grid = static_cast<unsigned>((rows + 3) / 4);
    const bool wide = h->cfg.head_dim == 128;
    switch (h->cfg.dtype) {
        case SISO_BF16:
            if (wide) kva::attention_rows_kernel<SISO_BF16, 128><<<grid, 128, 0, s>>>(g, h->status);
            else kva::attention_rows_kernel<SISO_BF16, 64><<<grid, 128, 0, s>>>(g, h->status);
            break;
        case SISO_E4M3:
            if (wide) kva::attention_rows_kernel<SISO_E4M3, 128><<<grid, 128, 0, s>>>(g, h->status);
            else kva::attention_rows_kernel<SISO_E4M3, 64><<<grid, 128, 0, s>>>(g, h->status);
            break;
        default:
            if (wide) kva::attention_rows_kernel<SISO_I8, 128><<<grid, 128, 0, s>>>(g, h->status);
            else kva::attention_rows_kernel<SISO_I8, 64><<<grid, 128, 0, s>>>(g, h->status);
    }
    SISO_CUDA(cudaGetLastError());
    return SISO_OK;
}

}  // namespace siso
