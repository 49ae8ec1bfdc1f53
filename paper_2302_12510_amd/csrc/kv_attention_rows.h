// Rows of queries in registers and their running results: shared by the kernels of the attention over the cache.
#pragma once
#include "kv_attention.h"
#include "kv_codec.h"

namespace dybit {
namespace kv {

constexpr float kLargeP = 16384.0f;                     // 2^14: what the largest probability times scale is brought to
constexpr float kFirstRef = 7.88860905e-31f;            // 2^-100: the reference of the values' scales before any is seen

__device__ __forceinline__ void load_query(const Phase &p, int64_t at, float (&x)[8])
{
    if (p.type == DYBIT_F32) {
        const float *q = (const float *)p.q + at;
        if (p.q_vectors) heads::Pack<float, 8>::load(q, x);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = q[i];
    } else if (p.type == DYBIT_F16) {
        const _Float16 *q = (const _Float16 *)p.q + at;
        if (p.q_vectors) heads::Pack<_Float16, 8>::load(q, x);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)q[i];
    } else {
        const __bf16 *q = (const __bf16 *)p.q + at;
        if (p.q_vectors) heads::Pack<__bf16, 8>::load(q, x);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)q[i];
    }
}

template <int N>
__device__ __forceinline__ void store_result(const Phase &p, int64_t at, const float (&x)[N])
{
    if (p.type == DYBIT_F32) {
        float *o = (float *)p.out + at;
        if (p.out_vectors) heads::Pack<float, N>::store(o, x);
        else
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = x[i];
    } else if (p.type == DYBIT_F16) {
        _Float16 *o = (_Float16 *)p.out + at;
        if (p.out_vectors) heads::Pack<_Float16, N>::store(o, x);
        else
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = (_Float16)x[i];
    } else {
        __bf16 *o = (__bf16 *)p.out + at;
        if (p.out_vectors) heads::Pack<__bf16, N>::store(o, x);
        else
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = (__bf16)x[i];
    }
}

// 16 rows of queries as operands, and what their scores are multiplied by.
template <int D, int TERMS>
struct Rows {
    f16x8 q[TERMS][D / 32];
    float factor;
    int seen;                                            // keys that this lane's row sees
    int64_t row;                                         // token * query heads + head; -1: no row
};

template <int KB, int D, int TERMS>
__device__ __forceinline__ void load_rows(const Phase &p, const Segment &g, int head, int64_t first_row, int lane, Rows<D, TERMS> &r)
{
    const int64_t n = first_row + (lane & 15);
    const int i = (int)(n / p.group), h = head * p.group + (int)(n - (int64_t)i * p.group);
    const bool real = i < g.count;
    const int64_t token = g.first + i;
    r.row = real ? token * (p.kv_heads * p.group) + h : -1;
    r.seen = real ? visible(p, g, i) : 0;
    float x[D / 32][8];
    float mx = 0.0f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[j][e] = 0.0f;
        if (real) load_query(p, token * p.q_token + h * p.q_head + (D / 4) * (lane >> 4) + 8 * j, x[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf(x[j][e]));
    }
    mx = max_over_groups(mx);
    u32 e = __float_as_uint(mx) >> 23;
    e = e == 255u ? 127u + 14u : e < 15u ? 15u : e;      // infinities stay infinite
    const float up = __uint_as_float((254u + 14u - e) << 23);
    r.factor = p.scale * __uint_as_float((e - 14u) << 23) * fold<KB>();
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int i8 = 0; i8 < 8; ++i8) {
            const float y = x[j][i8] * up;
            const _Float16 hi = (_Float16)y;
            r.q[0][j][i8] = hi;
            if constexpr (TERMS == 2) r.q[1][j][i8] = (_Float16)(y - (float)hi);
        }
}

// Running state of 16 rows.
template <int D>
struct State {
    f32x4 o[D / 16];
    float m, l;
};

// A row's result, or its part of one: a lane has dims (D / 16) (4 g4 + i) + j of its row.
template <int D>
__device__ __forceinline__ void write_row(const Phase &p, int64_t row, int slot, int g4, const State<D> &st)
{
    if (p.part_out) {
        const int64_t at = row * p.slots + p.slot0 + slot;
        if (g4 == 0) *reinterpret_cast<float2 *>(p.part_stat + 2 * at) = float2{st.m, st.l};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[D / 16];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) x[j] = st.o[j][i];
            heads::Pack<float, D / 16>::store(p.part_out + at * D + (D / 16) * (4 * g4 + i), x);
        }
    } else {
        const int heads_q = p.kv_heads * p.group;
        const int64_t token = row / heads_q;
        const int64_t at = token * p.out_token + (row - token * heads_q) * p.out_head;
        const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;                  // a row that sees nothing: zeros
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[D / 16];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) x[j] = st.o[j][i] * inv;
            store_result<D / 16>(p, at + (D / 16) * (4 * g4 + i), x);
        }
    }
}

}  // namespace kv
}  // namespace dybit
