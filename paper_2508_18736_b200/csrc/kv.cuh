// Internal declarations of the paged key/value cache: the handle, the device view that kernels get, and the code that
// turns 8-bit codes into values.
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace siso {

constexpr int kKvMaxDim = 256;

// What kernels see of the pages.  Strides in elements; the same for keys and values.
struct KvView {
    void *k, *v;
    uint8_t *k_exp, *v_exp;        // [n_layers, n_pages, n_kv_heads, page_size], 8-bit caches only
    long long n_pages, stride_page, stride_token, stride_head;
    int page_size, n_kv_heads, head_dim;
};

struct Kv {
    siso_kv_config_t cfg;
    int sm_count;
    void *ws;                      // scratch, grown on demand
    size_t ws_bytes;
    int *status;                   // device status word (first error wins)
    CUtensorMap map_k, map_v;      // (d, head, token, page, layer), for attention: head_dim 64 or 128
    int box;                       // tokens of their boxes: the largest power of two that divides the page and 128
    uint32_t attr_set;             // attention kernels that have been given their shared memory
};

inline int kv_elem_bytes(int dtype) { return dtype == SISO_BF16 ? 2 : 1; }

// Makes a device the calling thread's for as long as this lives, then the one that was
class OnDevice {
    int before_ = 0, device_;
    cudaError_t error_;

public:
    explicit OnDevice(int device) : device_(device) {
        error_ = cudaGetDevice(&before_);
        if (error_ == cudaSuccess && before_ != device_) error_ = cudaSetDevice(device_);
    }
    ~OnDevice() {
        if (error_ == cudaSuccess && before_ != device_) cudaSetDevice(before_);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
    cudaError_t error() const { return error_; }
};

// the pages of one layer
inline KvView kv_view(const Kv *h, int layer) {
    const siso_kv_config_t &g = h->cfg;
    const long long off = static_cast<long long>(layer) * g.stride_layer * kv_elem_bytes(g.dtype);
    const long long exps = static_cast<long long>(layer) * g.n_pages * g.n_kv_heads * g.page_size;
    KvView w;
    w.k = static_cast<char *>(g.d_k) + off;
    w.v = static_cast<char *>(g.d_v) + off;
    w.k_exp = g.d_k_exp ? g.d_k_exp + exps : nullptr;
    w.v_exp = g.d_v_exp ? g.d_v_exp + exps : nullptr;
    w.n_pages = g.n_pages;
    w.stride_page = g.stride_page;
    w.stride_token = g.stride_token;
    w.stride_head = g.stride_head;
    w.page_size = g.page_size;
    w.n_kv_heads = g.n_kv_heads;
    w.head_dim = g.head_dim;
    return w;
}

siso_status_t launch_kv_attention(Kv *h, const siso_attention_t *a, cudaStream_t s);
namespace kva { siso_status_t launch_wait_timeout(Kv *h, cudaStream_t s); }

#ifdef __CUDACC__
// Launches a kernel that may be set up while the one before it in the stream still runs (programmatic dependent launch).  It calls
// wait_for_earlier() before it touches memory.
template <typename... Params, typename... Given>
inline siso_status_t launch_early(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t s, const Given &...given) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SISO_CUDA(cudaLaunchKernelEx(&cfg, kernel, given...));
    return SISO_OK;
}
// Waits until the kernels before this one in the stream are complete and their writes visible.
__device__ __forceinline__ void wait_for_earlier() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Lets a kernel that was launched early be set up.  That happens once every CTA of this one has come here, so all have their places
// and none waits for room that the next kernel has taken.
__device__ __forceinline__ void dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// 2^(byte - 127) of a stored row; 255 marks a row that held a non-finite value
__device__ __forceinline__ float kv_scale(uint32_t byte) {
    return byte == 255u ? __uint_as_float(0x7FC00000u) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}
__device__ __forceinline__ uint32_t mul2_bf16(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t sub2_bf16(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Codes of one row as bf16, exactly: c 2^(byte - 127) has at most 8 significant bits.  e4m3: sign, exponent and mantissa moved to their places
// give the value times 2^-120, subnormal codes too, and the factor makes up for it.  i8: the low 7 bits as the mantissa of 128 + u,
// less 128 or, for negative codes, 256.
template <int KIND> struct CodeScale {
    uint32_t factor, more;                 // a second factor where 2^(byte - 7) itself is beyond bf16
    __device__ __forceinline__ explicit CodeScale(int byte) {
        const int field = KIND == SISO_E4M3 ? byte + 120 : byte;
        factor = (byte == 255 ? 0x7FC0u : field == 0 ? 0x0040u : static_cast<uint32_t>(min(field, 254)) << 7) * 0x10001u;
        more = KIND == SISO_E4M3 && byte > 134 && byte < 255 ? (static_cast<uint32_t>(field - 254 + 127) << 7) * 0x10001u : 0u;
    }
    // codes 0, 2 and 1, 3 of a word
    __device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) const {
        if constexpr (KIND == SISO_E4M3) {
            lo = mul2_bf16(((w << 4) & 0x07F007F0u) | ((w << 8) & 0x80008000u), factor);
            hi = mul2_bf16(((w >> 4) & 0x07F007F0u) | (w & 0x80008000u), factor);
            if (more) {
                lo = mul2_bf16(lo, more);
                hi = mul2_bf16(hi, more);
            }
        } else {
            const uint32_t x = w >> 8;
            lo = mul2_bf16(sub2_bf16((w & 0x007F007Fu) | 0x43004300u, (w & 0x00800080u) | 0x43004300u), factor);
            hi = mul2_bf16(sub2_bf16((x & 0x007F007Fu) | 0x43004300u, (x & 0x00800080u) | 0x43004300u), factor);
        }
    }
};
// value of one code.  e4m3: sign, 4 exponent and 3 mantissa bits moved to their places in a float give the value times
// 2^-120, subnormal codes too
template <int KIND> __device__ __forceinline__ float kv_code(uint32_t b, float scale) {
    if constexpr (KIND == SISO_E4M3)
        return __uint_as_float(((b & 0x80u) << 24) | ((b & 0x7Fu) << 20)) * __uint_as_float(247u << 23) * scale;
    return static_cast<float>(static_cast<int>(b << 24) >> 24) * scale;
}
#endif

}  // namespace siso

struct siso_kv : public siso::Kv {};
