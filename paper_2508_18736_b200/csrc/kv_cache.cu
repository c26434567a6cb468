// Paged key/value cache: the handle, quantisation of new rows as they are written, and reading rows back.
//
// A row is the head_dim values of one token in one kv head, of K or of V.  In an 8-bit cache it is kept as codes c_i and one
// exponent byte e + 127:
//     a = max |x_i|,   e = the smallest whole number >= -127 with a <= M 2^e   (M = 448 for e4m3, 127 for i8)
//     c_i = x_i 2^-e rounded to the nearest code, ties to even;   read back: c_i 2^e
// The scale is a power of two on purpose.  Both multiplications are then exact, so a code is rounded once, and c 2^e needs
// at most 8 significant bits: it is a bf16 value, which attention multiplies as it is.  The price is a step up to twice as
// coarse as a / M would give for i8 (e4m3 loses nothing but range at the bottom).  A row with a NaN or an infinity gets the
// byte 255 and reads back as NaN throughout.
//
// Both kernels move bytes: they are bound by HBM for prompts and by latency for a step's few tokens.  G lanes own the rows of one
// token with 16 values each, so the maximum takes log2 G shuffles; they look the slot up once and go through heads, U rows in
// flight.  16385 tokens x 8 x 128 bf16 into an 8-bit cache and back: 39.6 us together, 5 TB/s, issue at 60 % (one step's 48 tokens: 4 us).
// (With 8 values a lane what a row costs beside its values made issue the limit: 23 us and 19 us for 16385 tokens x 8 x 128.)
#include <cuda_fp8.h>

#include <cstring>
#include <new>

#include "kv.cuh"

namespace siso {
namespace kvc {

constexpr int THREADS = 256;
constexpr int U = 2;                     // (16385 x 8 x 128: 39.1 us, four 37.6; but 1000 tokens 6.3 and 8.0, fp32 rows 30.5 and 46.6)

struct Rows {                     // n tokens x heads rows of the caller's K and V
    void *k, *v;
    long long n, stride_token, stride_head;
};

template <typename T> struct Vec8;             // 8 consecutive values of the caller's type
template <> struct Vec8<__nv_bfloat16> {
    uint4 r;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = r; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        r = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void clear() { r = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void as_bf16(__nv_bfloat16 *p) const { store(p); }
    // bits of the largest magnitude, two values at a time: 16-bit patterns order like the values too
    __device__ __forceinline__ uint32_t largest() const {
        const uint32_t m = 0x7FFF7FFFu, x = __vmaxu2(__vmaxu2(r.x & m, r.y & m), __vmaxu2(r.z & m, r.w & m));
        return max(x << 16, x & 0xFFFF0000u);
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = reinterpret_cast<const float4 *>(p)[0]; b = reinterpret_cast<const float4 *>(p)[1]; }
    __device__ __forceinline__ void store(float *p) const { reinterpret_cast<float4 *>(p)[0] = a; reinterpret_cast<float4 *>(p)[1] = b; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&x)[8]) { a = make_float4(x[0], x[1], x[2], x[3]); b = make_float4(x[4], x[5], x[6], x[7]); }
    __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void as_bf16(__nv_bfloat16 *p) const {
        float x[8];
        get(x);
        Vec8<__nv_bfloat16> o;
        o.set(x);
        o.store(p);
    }
    __device__ __forceinline__ uint32_t largest() const {
        float x[8];
        get(x);
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
        return top;
    }
};

// exponent byte of a row whose largest magnitude is `a` (NaN where the row is not finite): M = top_mant 2^top_exp as float bits
template <int KIND> __device__ __forceinline__ int exponent_of(float a) {
    constexpr uint32_t top = KIND == SISO_E4M3 ? 0x43E00000u /* 448 */ : 0x42FE0000u /* 127 */;
    const uint32_t u = __float_as_uint(a);
    int e = static_cast<int>(u >> 23) - static_cast<int>(top >> 23) + ((u & 0x7FFFFFu) > (top & 0x7FFFFFu) ? 1 : 0);
    return max(e, -127);          // zero and subnormal rows end here too
}
// 2^-e for e in [-127, 122] (e4m3 goes to 120)
__device__ __forceinline__ float inverse_scale(int e) { return __uint_as_float(static_cast<uint32_t>(127 - e) << 23); }

template <int KIND> __device__ __forceinline__ uint2 encode8(const float (&x)[8], float inv) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (KIND == SISO_E4M3) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * h] * inv, x[4 * h + 1] * inv), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * h + 2] * inv, x[4 * h + 3] * inv), __NV_SATFINITE, __NV_E4M3);
            w[h] = lo | (hi << 16);
        } else {
            // 1.5 2^23 added: rounded to a whole number (nearest, ties to even) that stands in the low bits, negative ones in two's complement
            uint32_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(fmaf(x[4 * h + i], inv, 12582912.f));
            w[h] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
        }
    }
    return make_uint2(w[0], w[1]);
}
template <int KIND> __device__ __forceinline__ void decode8(uint2 c, float scale, float (&x)[8]) {
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = kv_code<KIND>((w[i >> 2] >> (8 * (i & 3))) & 0xFFu, scale);
}

template <int KIND, typename T, int G, bool READ>
__global__ void __launch_bounds__(THREADS)
kv_rows_kernel(KvView kv, Rows rows, const long long *__restrict__ slots, int heads_each) {
    wait_for_earlier();
    dependents_may_start();
    const int sub = threadIdx.x % G, d = sub * 8;          // a lane has the values d .. d + 7 and d + 8 G .. d + 8 G + 7: neighbours load neighbours
    const bool mine[2] = {d < kv.head_dim, d + 8 * G < kv.head_dim};
    const bool is_v = blockIdx.y != 0;
    char *pages = static_cast<char *>(is_v ? kv.v : kv.k);
    uint8_t *exps = is_v ? kv.v_exp : kv.k_exp;
    constexpr int EB = KIND == SISO_BF16 ? 2 : 1;
    const long long tok = static_cast<long long>(blockIdx.x) * (THREADS / G) + threadIdx.x / G;
    const int h0 = blockIdx.z * heads_each, h1 = min(kv.n_kv_heads, h0 + heads_each);
    // the token's row of head h0: in the caller's rows, in the pages, its exponent
    T *ext = static_cast<T *>(is_v ? rows.v : rows.k) + tok * rows.stride_token + h0 * rows.stride_head + d;
    const bool there = tok < rows.n;
    bool in_pool = false;
    if (there) {
        const long long slot = slots[tok];
        const long long page = slot < 0 ? -1 : (slot <= 0xFFFFFFFFll ? static_cast<uint32_t>(slot) / static_cast<uint32_t>(kv.page_size) : slot / kv.page_size);
        if (page >= 0 && page < kv.n_pages) {
            const int t = static_cast<int>(slot - page * kv.page_size);
            in_pool = true;
            pages += (page * kv.stride_page + t * kv.stride_token + h0 * kv.stride_head + d) * EB;
            exps += (page * kv.n_kv_heads + h0) * kv.page_size + t;
        }
    }
    for (int h = h0; h < h1; h += U) {
        if constexpr (!READ) {
            Vec8<T> in[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (mine[x] && there && h + u < h1) in[u][x].load(ext + u * rows.stride_head + 8 * G * x);
                    else in[u][x].clear();
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool store = in_pool && h + u < h1;
                char *dst = pages + u * kv.stride_head * EB;
                if constexpr (KIND == SISO_BF16) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (store && mine[x]) in[u][x].as_bf16(reinterpret_cast<__nv_bfloat16 *>(dst) + 8 * G * x);
                } else {
                    // magnitudes order like their bits, with infinities and NaN above every finite value
                    uint32_t top = max(in[u][0].largest(), in[u][1].largest());
#pragma unroll
                    for (int o = 1; o < G; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                    const bool finite = top < 0x7F800000u;
                    const int e = finite ? exponent_of<KIND>(__uint_as_float(top)) : 0;
                    const float inv = inverse_scale(e);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (!finite) in[u][x].clear();
                        float y[8];
                        in[u][x].get(y);
                        if (store && mine[x]) *reinterpret_cast<uint2 *>(dst + 8 * G * x) = encode8<KIND>(y, inv);
                    }
                    if (store && sub == 0) exps[u * kv.page_size] = finite ? static_cast<uint8_t>(e + 127) : 255;
                }
            }
        } else {
            Vec8<__nv_bfloat16> wide[U][2];
            uint2 codes[U][2];
            uint32_t e[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                e[u] = 127u;
                if (KIND != SISO_BF16 && in_pool && h + u < h1) e[u] = exps[u * kv.page_size];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const char *src = pages + (u * kv.stride_head + 8 * G * x) * EB;
                    wide[u][x].clear();
                    codes[u][x] = make_uint2(0u, 0u);
                    if (!mine[x] || !in_pool || h + u >= h1) continue;
                    if constexpr (KIND == SISO_BF16) wide[u][x].load(reinterpret_cast<const __nv_bfloat16 *>(src));
                    else codes[u][x] = *reinterpret_cast<const uint2 *>(src);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!there || h + u >= h1) continue;
                const CodeScale<KIND> scale(static_cast<int>(e[u]));
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!mine[x]) continue;
                    T *dst = ext + u * rows.stride_head + 8 * G * x;
                    if constexpr (KIND == SISO_BF16 && sizeof(T) == 2) wide[u][x].store(dst);
                    else if constexpr (KIND != SISO_BF16 && sizeof(T) == 2) {
                        uint32_t w[4];
                        scale.widen(codes[u][x].x, w[0], w[1]);
                        scale.widen(codes[u][x].y, w[2], w[3]);
                        *reinterpret_cast<uint4 *>(dst) = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[0], w[1], 0x7632),
                                                                    __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[2], w[3], 0x7632));
                    } else {
                        float y[8];
                        if constexpr (KIND == SISO_BF16) wide[u][x].get(y);
                        else decode8<KIND>(codes[u][x], kv_scale(e[u]), y);
                        Vec8<T> o;
                        o.set(y);
                        o.store(dst);
                    }
                }
            }
        }
        ext += U * rows.stride_head;
        pages += U * kv.stride_head * EB;
        exps += U * kv.page_size;
    }
}

template <int KIND, typename T, bool READ>
static siso_status_t run_rows(const KvView &kv, const Rows &rows, const long long *slots, int sm_count, cudaStream_t s) {
    const int g = kv.head_dim <= 64 ? 4 : kv.head_dim <= 128 ? 8 : 16;
    const long long blocks = (rows.n + THREADS / g - 1) / (THREADS / g);
    if (blocks > 0x7FFFFFFFll) return SISO_ERR_UNSUPPORTED;
    // a prompt's lanes go through all heads of their token; the few tokens of a step are spread over more CTAs, a head each
    const int heads_each = blocks >= sm_count ? kv.n_kv_heads : 1;
    const dim3 grid(static_cast<unsigned>(blocks), 2, static_cast<unsigned>((kv.n_kv_heads + heads_each - 1) / heads_each));
    if (g == 4) return launch_early(kv_rows_kernel<KIND, T, 4, READ>, grid, THREADS, 0, s, kv, rows, slots, heads_each);
    if (g == 8) return launch_early(kv_rows_kernel<KIND, T, 8, READ>, grid, THREADS, 0, s, kv, rows, slots, heads_each);
    return launch_early(kv_rows_kernel<KIND, T, 16, READ>, grid, THREADS, 0, s, kv, rows, slots, heads_each);
}
template <typename T, bool READ>
static siso_status_t run_kind(int kind, const KvView &kv, const Rows &rows, const long long *slots, int sm_count, cudaStream_t s) {
    return kind == SISO_E4M3 ? run_rows<SISO_E4M3, T, READ>(kv, rows, slots, sm_count, s)
         : kind == SISO_I8 ? run_rows<SISO_I8, T, READ>(kv, rows, slots, sm_count, s) : run_rows<SISO_BF16, T, READ>(kv, rows, slots, sm_count, s);
}

static bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <bool READ>
static siso_status_t rows_call(Kv *h, int layer, void *k, void *v, int dtype, long long n, long long stride_token, long long stride_head,
                               const int64_t *slots, cudaStream_t s) {
    if (!h || layer < 0 || layer >= h->cfg.n_layers || n < 0) return SISO_ERR_INVALID_ARG;
    if (dtype != SISO_F32 && dtype != SISO_BF16) return SISO_ERR_INVALID_ARG;
    if (n == 0) return SISO_OK;
    if (n == 1) stride_token = 0;                  // a dimension of one entry has no stride, whatever its tensor says
    if (h->cfg.n_kv_heads == 1) stride_head = 0;
    if (!k || !v || !slots || stride_token < 0 || stride_head < 0) return SISO_ERR_INVALID_ARG;
    const int elems16 = dtype == SISO_F32 ? 4 : 8;
    if (!aligned16(k) || !aligned16(v) || stride_token % elems16 != 0 || stride_head % elems16 != 0) return SISO_ERR_UNSUPPORTED;
    const OnDevice on(h->cfg.device);
    SISO_CUDA(on.error());
    const Rows rows{k, v, n, stride_token, stride_head};
    const KvView kv = kv_view(h, layer);
    const long long *sl = reinterpret_cast<const long long *>(slots);
    return dtype == SISO_F32 ? run_kind<float, READ>(h->cfg.dtype, kv, rows, sl, h->sm_count, s)
                             : run_kind<__nv_bfloat16, READ>(h->cfg.dtype, kv, rows, sl, h->sm_count, s);
}

// Tensor maps of the pages for attention: boxes of `box` tokens of one page and head, 128 bytes wide (64 where a row has no more),
// swizzled so that consecutive tokens start in different banks.
static siso_status_t encode_maps(Kv *h) {
    const siso_kv_config_t &g = h->cfg;
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult res;
    SISO_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &res));
    if (!fn || res != cudaDriverEntryPointSuccess) return check_cuda(cudaErrorNotSupported, "cuTensorMapEncodeTiled lookup");
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    const cuuint64_t eb = kv_elem_bytes(g.dtype), row = g.head_dim * eb;
    for (h->box = 128; g.page_size % h->box != 0;) h->box /= 2;
    const cuuint64_t dims[5] = {static_cast<cuuint64_t>(g.head_dim), static_cast<cuuint64_t>(g.n_kv_heads), static_cast<cuuint64_t>(g.page_size),
                                static_cast<cuuint64_t>(g.n_pages), static_cast<cuuint64_t>(g.n_layers)};
    // a dimension of one entry has no stride of its own
    const cuuint64_t strides[4] = {std::max<cuuint64_t>(g.stride_head * eb, 16), std::max<cuuint64_t>(g.stride_token * eb, 16),
                                   std::max<cuuint64_t>(g.stride_page * eb, 16), std::max<cuuint64_t>(g.stride_layer * eb, 16)};
    const cuuint32_t box[5] = {static_cast<cuuint32_t>(std::min<cuuint64_t>(row, 128) / eb), 1u, static_cast<cuuint32_t>(h->box), 1u, 1u};
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < 2; ++i) {
        const CUresult r = reinterpret_cast<Encode>(fn)(
            i ? &h->map_v : &h->map_k, eb == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, i ? g.d_v : g.d_k, dims, strides,
            box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, row >= 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            row >= 256 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : row >= 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r != CUDA_SUCCESS) return check_cuda(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    }
    return SISO_OK;
}

// whether attention can read these pages: its head sizes, and 16 bytes at a time
static bool attends(const siso_kv_config_t &g) {
    const int64_t elems16 = 16 / kv_elem_bytes(g.dtype);
    return (g.head_dim == 64 || g.head_dim == 128) && g.stride_layer % elems16 == 0 && g.stride_page % elems16 == 0 &&
           g.stride_token % elems16 == 0 && g.stride_head % elems16 == 0;
}

}  // namespace kvc
}  // namespace siso

using namespace siso;

extern "C" {

siso_status_t siso_kv_create(siso_kv_t **out, const siso_kv_config_t *cfg) {
    if (!out || !cfg) return SISO_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg->d_k || !cfg->d_v || cfg->n_layers < 1 || cfg->n_pages < 1 || cfg->n_pages >= (1ll << 31) || cfg->page_size < 1 ||
        cfg->n_kv_heads < 1 || cfg->head_dim < 1)
        return SISO_ERR_INVALID_ARG;
    if (cfg->dtype != SISO_BF16 && cfg->dtype != SISO_E4M3 && cfg->dtype != SISO_I8) return SISO_ERR_INVALID_ARG;
    const bool eight = cfg->dtype != SISO_BF16;
    if (eight != (cfg->d_k_exp != nullptr) || eight != (cfg->d_v_exp != nullptr)) return SISO_ERR_INVALID_ARG;
    if ((cfg->allocator.alloc == nullptr) != (cfg->allocator.free == nullptr)) return SISO_ERR_INVALID_ARG;
    if (cfg->page_size % 8 != 0 || cfg->page_size > 65536 || cfg->head_dim % 8 != 0 || cfg->head_dim > kKvMaxDim || cfg->n_kv_heads > 4096)
        return SISO_ERR_UNSUPPORTED;
    siso_kv_config_t own = *cfg;
    cfg = &own;
    // a dimension of one entry has no stride, whatever its tensor says
    if (cfg->n_layers == 1) own.stride_layer = 0;
    if (cfg->n_pages == 1) own.stride_page = 0;
    if (cfg->n_kv_heads == 1) own.stride_head = 0;
    const long long strides[] = {cfg->stride_layer, cfg->stride_page, cfg->stride_token, cfg->stride_head};
    for (long long st : strides) {
        if (st < 0) return SISO_ERR_INVALID_ARG;
        if (st % 8 != 0 || st >= (1ll << 38)) return SISO_ERR_UNSUPPORTED;
    }
    // entries that share their place: rows would be written over one another, and TMA takes no stride of 0
    if ((cfg->n_layers > 1 && cfg->stride_layer == 0) || (cfg->n_pages > 1 && cfg->stride_page == 0) || cfg->stride_token == 0 ||
        (cfg->n_kv_heads > 1 && cfg->stride_head == 0))
        return SISO_ERR_UNSUPPORTED;
    if (!kvc::aligned16(cfg->d_k) || !kvc::aligned16(cfg->d_v) || !kvc::aligned16(cfg->d_k_exp) || !kvc::aligned16(cfg->d_v_exp))
        return SISO_ERR_UNSUPPORTED;
    int n_dev = 0;
    SISO_CUDA(cudaGetDeviceCount(&n_dev));
    if (cfg->device < 0 || cfg->device >= n_dev) return SISO_ERR_INVALID_ARG;
    const OnDevice on(cfg->device);
    SISO_CUDA(on.error());
    int major = 0, sms = 0;
    SISO_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, cfg->device));
    SISO_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, cfg->device));
    if (major != 10) return SISO_ERR_UNSUPPORTED;
    siso_kv *h = new (std::nothrow) siso_kv();
    if (!h) return SISO_ERR_OOM;
    memset(static_cast<Kv *>(h), 0, sizeof(Kv));
    h->cfg = *cfg;
    if (!cfg->allocator.alloc) h->cfg.allocator = default_allocator();
    h->sm_count = sms;
    if (kvc::attends(h->cfg)) {
        const siso_status_t st = kvc::encode_maps(h);
        if (st != SISO_OK) { delete h; return st; }
    }
    h->status = static_cast<int *>(h->cfg.allocator.alloc(256, nullptr, h->cfg.allocator.ctx));
    if (!h->status) { delete h; return SISO_ERR_OOM; }
    cudaError_t e = cudaMemset(h->status, 0, 256);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) { siso_kv_destroy(h); return check_cuda(e, "key/value cache initialisation"); }
    *out = h;
    return SISO_OK;
}

siso_status_t siso_kv_destroy(siso_kv_t *h) {
    if (!h) return SISO_ERR_INVALID_ARG;
    const OnDevice on(h->cfg.device);
    cudaDeviceSynchronize();
    if (h->ws) h->cfg.allocator.free(h->ws, h->cfg.allocator.ctx);
    if (h->status) h->cfg.allocator.free(h->status, h->cfg.allocator.ctx);
    delete h;
    return SISO_OK;
}

siso_status_t siso_kv_write(siso_kv_t *h, int32_t layer, const void *d_k, const void *d_v, int32_t dtype, int64_t n_tokens,
                            int64_t stride_token, int64_t stride_head, const int64_t *d_slots, void *stream) {
    return kvc::rows_call<false>(h, layer, const_cast<void *>(d_k), const_cast<void *>(d_v), dtype, n_tokens, stride_token, stride_head,
                                 d_slots, static_cast<cudaStream_t>(stream));
}

siso_status_t siso_kv_read(siso_kv_t *h, int32_t layer, void *d_k, void *d_v, int32_t dtype, int64_t n_tokens, int64_t stride_token,
                           int64_t stride_head, const int64_t *d_slots, void *stream) {
    return kvc::rows_call<true>(h, layer, d_k, d_v, dtype, n_tokens, stride_token, stride_head, d_slots, static_cast<cudaStream_t>(stream));
}

siso_status_t siso_kv_attention(siso_kv_t *h, const siso_attention_t *args, void *stream) {
    const siso_attention_t *a = args;
    if (!h || !a || a->n_tokens < 0 || a->n_seqs < 0 || a->layer < 0 || a->layer >= h->cfg.n_layers) return SISO_ERR_INVALID_ARG;
    if (a->n_heads < 1 || a->n_heads % h->cfg.n_kv_heads != 0 || a->window < 0 || a->max_q < 0 || a->max_pages < 0) return SISO_ERR_INVALID_ARG;
    if ((a->flags & ~SISO_ATTN_CAUSAL) != 0u || !(a->scale == a->scale)) return SISO_ERR_INVALID_ARG;
    if (a->n_tokens == 0 || a->n_seqs == 0) return SISO_OK;
    if (!a->d_q || !a->d_out || !a->d_cu_q || !a->d_kv_len || (a->max_pages > 0 && !a->d_pages) || a->pages_stride < 0) return SISO_ERR_INVALID_ARG;
    siso_attention_t own = *args;
    a = &own;
    if (a->n_tokens == 1) own.q_stride_token = own.out_stride_token = 0;       // (one entry: no stride)
    if (a->n_heads == 1) own.q_stride_head = own.out_stride_head = 0;
    const int64_t strides[] = {a->q_stride_token, a->q_stride_head, a->out_stride_token, a->out_stride_head};
    for (int64_t st : strides) {
        if (st < 0) return SISO_ERR_INVALID_ARG;
        if (st % 8 != 0) return SISO_ERR_UNSUPPORTED;
    }
    if (!kvc::aligned16(a->d_q) || !kvc::aligned16(a->d_out)) return SISO_ERR_UNSUPPORTED;
    if (!kvc::attends(h->cfg)) return SISO_ERR_UNSUPPORTED;
    if (a->n_tokens >= ((1ll << 31) - 256) / a->n_heads || static_cast<int64_t>(a->max_pages) * h->cfg.page_size >= (1ll << 31) - 65536) return SISO_ERR_UNSUPPORTED;
    const OnDevice on(h->cfg.device);
    SISO_CUDA(on.error());
    return launch_kv_attention(h, a, static_cast<cudaStream_t>(stream));
}

siso_status_t siso_kv_selftest_wait_timeout(siso_kv_t *h, void *stream) {
    if (!h) return SISO_ERR_INVALID_ARG;
    const OnDevice on(h->cfg.device);
    SISO_CUDA(on.error());
    return kva::launch_wait_timeout(h, static_cast<cudaStream_t>(stream));
}

siso_status_t siso_kv_sync_status(siso_kv_t *h, void *stream) {
    if (!h) return SISO_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const OnDevice on(h->cfg.device);
    SISO_CUDA(on.error());
    int st = 0;
    SISO_CUDA(cudaMemcpyAsync(&st, h->status, sizeof(int), cudaMemcpyDeviceToHost, s));
    SISO_CUDA(cudaMemsetAsync(h->status, 0, sizeof(int), s));
    SISO_CUDA(cudaStreamSynchronize(s));
    return static_cast<siso_status_t>(st);
}

}  // extern "C"
