// Filling and moving the key/value cache: new tokens encoded into their pages, pages copied to other pages.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kv_cache.h"
#include "requant.h"

namespace dybit {
namespace kv {

constexpr int kThreads = 256;

// ---- append ---------------------------------------------------------------------------------------------------------------------
// A head's D elements lie in D / 8 lanes, eight each: the maximum goes round those lanes, each encodes its eight and stores one word
// (4 bits) or two.  Before the encoder the head and its scale are multiplied by the power of two that brings the scale into [1, 2):
// exact but for elements that underflow, whose code is 0 either way, and so any normal scale takes the encoder's one path.
// Bound by memory: 16383 tokens of 8 heads of 128, fp32 to keys of 8 bits and values of 4, 161 MB in 34.0 us, 4.7 TB/s (a device copy: 5.1).
struct AppendArgs {
    const void *x[2];
    int64_t token_stride[2], head_stride[2];
    uint8_t *codes[2];
    float *scales[2];
    int32_t bits[2];
    const int64_t *slots;
    int64_t rows, places;               // tokens x heads; places in the pool
    int32_t heads, page_shift;
    int *err;
};

// V: elements of one access (8, or 1 where a head does not start on a multiple of eight elements).
template <class T, int D, int V>
__global__ __launch_bounds__(kThreads) void append_kernel(const AppendArgs p)
{
    constexpr int LANES = D / 8;
    const int kv = blockIdx.y, lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;
    const bool real = row < p.rows;
    const int64_t t = real ? row / p.heads : 0;
    const int h = real ? (int)(row - t * p.heads) : 0;
    const int64_t slot = real ? p.slots[t] : -1;
    const bool in = slot >= 0 && slot < p.places;
    if (slot >= p.places && lane == 0) *p.err = DYBIT_ERR_INVALID_ARG;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.0f;
    if (in) {
        const T *from = (const T *)p.x[kv] + t * p.token_stride[kv] + h * p.head_stride[kv] + lane * 8;
        if constexpr (V == 8) heads::Pack<T, 8>::load(from, x);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)from[i];
    }
    float mx = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(x[i]));                  // a NaN loses to any number
#pragma unroll
    for (int off = 1; off < LANES; off <<= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    if (!in) return;
    const int bits = p.bits[kv], m = bits - 1;
    float s = mx == 0.0f ? 1.0f : mx * __uint_as_float((uint32_t)(127 - (m - 1)) << 23);
    const uint32_t e = __float_as_uint(s) >> 23;
    const bool flat = e == 0u;                                                 // a subnormal scale: stored as zeros
    const bool infinite = e == 255u;
    if (flat) s = 1.0f;
    const float p2 = __uint_as_float((254u - (flat || infinite ? 127u : e)) << 23);
    const float s2 = infinite ? 1.0f : s * p2;
    const float keep = flat || infinite ? 0.0f : p2;
    const Requant r = make_requant(s2, 1.0f / s2, bits, 1);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = keep == 0.0f ? 0u : requant_code(x[i] * keep, r);
    const int64_t place = (((slot >> p.page_shift) * p.heads + h) << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
    if (bits == 8) {
        uint2 w;
        w.x = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
        w.y = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
        *reinterpret_cast<uint2 *>(p.codes[kv] + place * D + lane * 8) = w;
    } else {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= c[i] << (4 * i);
        *reinterpret_cast<uint32_t *>(p.codes[kv] + place * (D / 2) + lane * 4) = w;
    }
    if (lane == 0) {
        p.scales[kv][place] = infinite ? __builtin_nanf("") : s;
        if (infinite) *p.err = DYBIT_ERR_BAD_SCALE;
    }
}

template <class T>
void launch_append(const AppendArgs &p, int D, bool vectors, hipStream_t st)
{
    const int per_block = kThreads / (D / 8);
    const dim3 grid((unsigned)((p.rows + per_block - 1) / per_block), 2), block(kThreads);
#define DYBIT_AP(D) if (vectors) hipLaunchKernelGGL((append_kernel<T, D, 8>), grid, block, 0, st, p); \
                    else hipLaunchKernelGGL((append_kernel<T, D, 1>), grid, block, 0, st, p)
    if (D == 64) { DYBIT_AP(64); }
    else if (D == 128) { DYBIT_AP(128); }
    else { DYBIT_AP(256); }
#undef DYBIT_AP
}

// ---- copies of pages -------------------------------------------------------------------------------------------------------------
// A page of a layer is four runs of whole 16-byte words (codes and scales of keys and of values); a workgroup moves a part of it,
// every lane kUnroll words that are all requested before the first is stored.  Bound by memory: 511 pages in 16 layers, 2.21 GB, in
// 438 us, 5.05 TB/s, a device copy's rate.
struct CopyArgs {
    uint8_t *base[4];
    int64_t layer_bytes[4];             // from a layer's run to the next layer's
    int32_t words[4];                   // 16-byte words of a page's run
    const int32_t *src, *dst;
    int64_t pages;
    int32_t layers, parts, total;       // workgroups per page and layer; words of a page
    int *err;
};
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kUnroll = 4;

__global__ __launch_bounds__(kThreads) void copy_pages_kernel(const CopyArgs p)
{
    const uint32_t per_page = (uint32_t)p.layers * (uint32_t)p.parts;
    const uint32_t i = blockIdx.x / per_page, rest = blockIdx.x - i * per_page;
    const uint32_t layer = rest / (uint32_t)p.parts, part = rest - layer * (uint32_t)p.parts;
    const int64_t from = p.src[i], to = p.dst[i];
    if (from < 0 || to < 0 || from >= p.pages || to >= p.pages) {
        if (threadIdx.x == 0) *p.err = DYBIT_ERR_INVALID_ARG;
        return;
    }
    u32x4 v[kUnroll];
    u32x4 *out[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
        int w = (int)(part * kUnroll + k) * kThreads + (int)threadIdx.x;
        out[k] = nullptr;
        if (w < p.total) {
            int run = 0;
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (run == j && w >= p.words[j]) { w -= p.words[j]; run = j + 1; }
            uint8_t *base = p.base[run] + layer * p.layer_bytes[run] + (int64_t)w * 16;
            const int64_t page_bytes = (int64_t)p.words[run] * 16;
            v[k] = *reinterpret_cast<const u32x4 *>(base + from * page_bytes);
            out[k] = reinterpret_cast<u32x4 *>(base + to * page_bytes);
        }
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
        if (out[k]) *out[k] = v[k];
}

}  // namespace kv
}  // namespace dybit

extern "C" dybit_status dybit_kv_append(dybit_heads keys, dybit_heads values, const int64_t *slots, dybit_kv_cache cache, dybit_stream stream)
{
    using namespace dybit;
    dybit_status st = kv::check(cache);
    if (st != DYBIT_OK) return st;
    for (const dybit_heads *h : {&keys, &values}) {
        st = heads::check(*h);
        if (st != DYBIT_OK) return st;
        if (h->heads != cache.heads || h->head_dim != cache.head_dim || !heads::same_shape(*h, keys)) return DYBIT_ERR_INVALID_ARG;
    }
    if (cache.layers != 1) return DYBIT_ERR_INVALID_ARG;
    if (keys.tokens == 0) return DYBIT_OK;
    if (!slots) return DYBIT_ERR_NULL;
    kv::AppendArgs p{};
    p.x[0] = keys.data; p.token_stride[0] = keys.token_stride; p.head_stride[0] = keys.head_stride;
    p.x[1] = values.data; p.token_stride[1] = values.token_stride; p.head_stride[1] = values.head_stride;
    p.codes[0] = cache.k_codes; p.scales[0] = cache.k_scales; p.bits[0] = cache.k_fmt.bits;
    p.codes[1] = cache.v_codes; p.scales[1] = cache.v_scales; p.bits[1] = cache.v_fmt.bits;
    p.slots = slots;
    p.rows = keys.tokens * keys.heads;
    p.places = cache.pages * cache.page_tokens;
    p.heads = cache.heads;
    p.page_shift = kv::log2_of(cache.page_tokens);
    if (p.rows > ((int64_t)0x7fffffff)) return DYBIT_ERR_INVALID_ARG;
    p.err = async_error_word();
    if (!p.err) return DYBIT_ERR_HIP;
    const bool vectors = heads::aligned(keys, 8) && heads::aligned(values, 8);
    switch (keys.type) {
        case DYBIT_F32: kv::launch_append<float>(p, cache.head_dim, vectors, (hipStream_t)stream); break;
        case DYBIT_F16: kv::launch_append<_Float16>(p, cache.head_dim, vectors, (hipStream_t)stream); break;
        default: kv::launch_append<__bf16>(p, cache.head_dim, vectors, (hipStream_t)stream); break;
    }
    return launch_status();
}

extern "C" dybit_status dybit_kv_copy_pages(dybit_kv_cache cache, const int32_t *src, const int32_t *dst, int64_t n, dybit_stream stream)
{
    using namespace dybit;
    const dybit_status st = kv::check(cache);
    if (st != DYBIT_OK) return st;
    if (n < 0 || n > cache.pages) return DYBIT_ERR_INVALID_ARG;
    if (n == 0 || cache.layers == 0) return DYBIT_OK;
    if (!src || !dst) return DYBIT_ERR_NULL;
    kv::CopyArgs p{};
    uint8_t *base[4] = {cache.k_codes, cache.v_codes, (uint8_t *)cache.k_scales, (uint8_t *)cache.v_scales};
    const int64_t places = (int64_t)cache.heads * cache.page_tokens;
    const int64_t bytes[4] = {places * cache.head_dim * cache.k_fmt.bits / 8, places * cache.head_dim * cache.v_fmt.bits / 8, places * 4, places * 4};
    int64_t total = 0;
    for (int j = 0; j < 4; ++j) {
        p.base[j] = base[j];
        p.words[j] = (int32_t)(bytes[j] / 16);
        p.layer_bytes[j] = bytes[j] * cache.pages;
        total += bytes[j] / 16;
    }
    const int64_t parts = (total + kv::kThreads * kv::kUnroll - 1) / (kv::kThreads * kv::kUnroll);
    if (total > 0x3fffffff || cache.layers * parts > 0x7fffffff) return DYBIT_ERR_INVALID_ARG;
    p.src = src; p.dst = dst; p.pages = cache.pages;
    p.layers = (int32_t)cache.layers; p.parts = (int32_t)parts; p.total = (int32_t)total;
    p.err = async_error_word();
    if (!p.err) return DYBIT_ERR_HIP;
    // a launch holds at most 2^23 workgroups of 256 threads here: longer lists go in several
    const int64_t per_launch = std::max<int64_t>(1, (int64_t)(1 << 23) / (cache.layers * parts));
    for (int64_t at = 0; at < n; at += per_launch) {
        p.src = src + at;
        p.dst = dst + at;
        const int64_t count = std::min(per_launch, n - at);
        hipLaunchKernelGGL(kv::copy_pages_kernel, dim3((unsigned)(count * cache.layers * parts)), dim3(kv::kThreads), 0, (hipStream_t)stream, p);
    }
    return launch_status();
}
