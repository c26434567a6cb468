// The weight that attention gives to each cached token, accumulated: for the eviction by it.
//
// Query i of a sequence (head g of the kv head's group) gives token j, if it sees it, exp(scale q.k_j - lse): its probability.  For each token and
// kv head the call takes w_j <- decay w_j + sum over queries and heads.  The statistics (lse) are the attention's, so one pass over the keys is all.
#include "kv_attention.cuh"

namespace siso {
namespace kvw {

struct Args {
    KvView kv;
    siso_weights_t a;
    int group;
    float scale_log2;
    int *status;
};

// A CTA per (tile of 128 tokens, kv head, sequence), a thread per token
template <int KIND, int D>
__global__ void __launch_bounds__(128)
weights_plain_kernel(const __grid_constant__ Args g) {
    __shared__ float q[8][D], shift[8];
    const int b = blockIdx.z, head = blockIdx.y;
    const int n = static_cast<int>(g.a.n_tokens), q0 = min(max(g.a.d_cu_q[b], 0), n), n_q = max(0, min(g.a.d_cu_q[b + 1], n) - q0);
    const int len = static_cast<int>(min(static_cast<long long>(max(g.a.d_kv_len[b], 0)), static_cast<long long>(g.a.max_pages) * g.kv.page_size));
    const bool causal = (g.a.flags & SISO_ATTN_CAUSAL) != 0u;
    if (n_q == 0) return;
    for (int j0 = blockIdx.x * 128; j0 < len; j0 += gridDim.x * 128) {
        const int j = j0 + threadIdx.x;
        int page = -1, tok = 0;
        if (j < len) {
            page = g.a.d_pages[b * g.a.pages_stride + j / g.kv.page_size];
            tok = j % g.kv.page_size;
            if (page < 0 || page >= g.kv.n_pages) { page = -1; set_status(g.status, SISO_ERR_INVALID_ARG); }
        }
        float k[D], sum = 0.f;
        const long long small = (static_cast<long long>(page) * g.kv.n_kv_heads + head) * g.kv.page_size + tok;
        if (page >= 0) {
            const long long at = page * g.kv.stride_page + tok * g.kv.stride_token + head * g.kv.stride_head;
            for (int d = 0; d < D; ++d) {
                if constexpr (KIND == SISO_BF16) k[d] = __bfloat162float(static_cast<const __nv_bfloat16 *>(g.kv.k)[at + d]);
                else k[d] = kv_code<KIND>(static_cast<const uint8_t *>(g.kv.k)[at + d], kv_scale(g.kv.k_exp[small]));
            }
        }
        for (int r0 = 0; r0 < n_q * g.group; r0 += 8) {
            __syncthreads();
            for (int x = threadIdx.x; x < 8 * D; x += 128) {
                const int r = r0 + x / D, i = r / g.group, h = head * g.group + r % g.group;
                if (r < n_q * g.group)
                    q[x / D][x % D] = __bfloat162float(static_cast<const __nv_bfloat16 *>(g.a.d_q)[(q0 + i) * g.a.q_stride_token + h * g.a.q_stride_head + x % D]);
                if (r < n_q * g.group && x % D == 0) shift[x / D] = g.a.d_lse[static_cast<long long>(q0 + i) * g.a.n_heads + h] * 1.4426950408889634f;
            }
            __syncthreads();
            for (int y = 0; y < 8 && r0 + y < n_q * g.group; ++y) {
                const int pos = kva::position(len, n_q, (r0 + y) / g.group);
                if (page < 0 || (causal && j > pos) || shift[y] == -INFINITY) continue;
                float s = 0.f;
                for (int d = 0; d < D; ++d) s += q[y][d] * k[d];
                sum += exp2f(s * g.scale_log2 - shift[y]);
            }
        }
        if (page >= 0) {
            float *w = g.a.d_weights + static_cast<long long>(g.a.layer) * g.kv.n_pages * g.kv.n_kv_heads * g.kv.page_size + small;
            *w = (j < len - n_q && g.a.decay != 0.f ? g.a.decay * *w : 0.f) + sum;
        }
    }
}

template <int KIND, int D> static siso_status_t run(Kv *h, const Args &g, cudaStream_t s) {
    const long long tiles = std::max<long long>(1, (static_cast<long long>(g.a.max_pages) * g.kv.page_size + 127) / 128);
    if (g.a.n_seqs > 65535) return SISO_ERR_UNSUPPORTED;
    weights_plain_kernel<KIND, D><<<dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(g.kv.n_kv_heads), static_cast<unsigned>(g.a.n_seqs)), 128, 0, s>>>(g);
    SISO_CUDA(cudaGetLastError());
    return SISO_OK;
}

}  // namespace kvw

siso_status_t launch_kv_weights(Kv *h, const siso_weights_t *a, cudaStream_t s) {
    using namespace kvw;
    Args g;
    g.kv = kv_view(h, a->layer);
    g.a = *a;
    g.group = a->n_heads / h->cfg.n_kv_heads;
    g.scale_log2 = a->scale * 1.4426950408889634f;
    g.status = h->status;
    const bool wide = h->cfg.head_dim == 128;
    switch (h->cfg.dtype) {
        case SISO_BF16: return wide ? run<SISO_BF16, 128>(h, g, s) : run<SISO_BF16, 64>(h, g, s);
        case SISO_E4M3: return wide ? run<SISO_E4M3, 128>(h, g, s) : run<SISO_E4M3, 64>(h, g, s);
        default: return wide ? run<SISO_I8, 128>(h, g, s) : run<SISO_I8, 64>(h, g, s);
    }
}

}  // namespace siso
