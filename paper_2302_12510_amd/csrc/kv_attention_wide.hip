// Attention over the cache of codes for many rows of queries (chunks of prompts, the queries of a group over its prefix); one build
// per pair of code widths (DYBIT_KV_K, DYBIT_KV_V).
//
// The arithmetic is kv_attention.hip's.  Here four waves hold 32 rows each and go through the same keys together: a step is 64 tokens,
// of which every wave decodes a quarter and leaves it in LDS as operands of the matrix instruction, 16 bytes a lane in lane order
// (no bank conflicts, no padding); all four read them all.  Decoding, some 2.5 instructions a code, is shared by 128 rows then.
// The next step's codes are requested before this step's products and decoded behind them, into the other half of the LDS.
#include <hip/hip_runtime.h>

#include "kv_attention_rows.h"

#ifndef DYBIT_KV_K
#define DYBIT_KV_K 8
#endif
#ifndef DYBIT_KV_V
#define DYBIT_KV_V 8
#endif

namespace dybit {
namespace kv {
namespace {

constexpr int KB = DYBIT_KV_K, VB = DYBIT_KV_V;
constexpr int kThreads = 256, kWaves = 4, kStep = 64, kBlocks = kStep / 16, NT = kWideRows / (16 * kWaves);

// What a wave decodes of a step: the keys of 16 tokens, half the dims of the values of 32, and the scales of 16.
template <int D>
struct Share {
    static constexpr int KW = D * KB / 128, VBYTES = D * VB / 256, VW = Values<VB, D / 32>::WORDS;
    u32 k[KW];
    u32 v[8][VW];
    float scale;                                         // lanes 0 to 15: of the keys, 16 to 31: of the values
    int valid;                                           // tokens of the block of 16 that count
};

template <int D, int BUFFERS>
struct Lds {
    f16x8 k[BUFFERS][kBlocks][D / 32][64];
    f16x8 v[BUFFERS][2][D / 16][64];
    float sk[BUFFERS][kStep], sv[BUFFERS][kStep];
    int valid[BUFFERS][kBlocks];
};

template <int D, int TERMS>
__global__ __launch_bounds__(kThreads, D * TERMS > 128 ? 1 : 2) void attention_wide_kernel(const Phase p)
{
    constexpr int BUFFERS = D == 256 ? 1 : 2;            // 64 KB a step of 256 dims
    __shared__ Lds<D, BUFFERS> lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g4 = lane >> 4;
    const int seg = (int)(blockIdx.x / (unsigned)p.kv_heads), head = (int)blockIdx.x - seg * p.kv_heads;
    const int row0 = (int)(gridDim.y - 1 - blockIdx.y) * (16 * NT * kWaves);       // causal: those with the most keys first
    const int slot = blockIdx.z;
    const Segment g = segment(p, seg);
    if (g.odd && head == 0 && row0 == 0 && slot == 0 && threadIdx.x == 0) *p.err = DYBIT_ERR_INVALID_ARG;
    if (row0 >= g.count * p.group) return;
    int last = (int)((unsigned)(row0 + 16 * NT * kWaves - 1) / (unsigned)p.group);
    last = last < g.count ? last : g.count - 1;
    const int lo = slot * p.chunk, most = visible(p, g, last);
    const int hi = most - lo < p.chunk ? most : lo + p.chunk;
    if (lo >= hi && p.part_out) return;

    Rows<D, TERMS> r[NT];
    State<D> st[NT];
    int least = 0x7fffffff;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        load_rows<KB, D, TERMS>(p, g, head, row0 + 16 * (NT * wave + t), lane, r[t]);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) st[t].o[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        st[t].m = -__builtin_inff();
        st[t].l = 0.0f;
        if (r[t].row >= 0) least = min(least, r[t].seen);
    }
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) least = min(least, __shfl_xor(least, off));
    least = __builtin_amdgcn_readfirstlane(least);

    const int steps = (hi - lo + kStep - 1) / kStep;
    const int32_t *table = p.tables + (int64_t)seg * p.table_width;
    const int vchunk = wave >> 1, vhalf = wave & 1;
    auto page_of = [&](int token) {                      // of a block of 16 tokens; -1: none that counts
        int id = -1;
        if (token < hi) {
            id = table[token >> p.page_shift];
            if (id < 0 || id >= p.pages) { id = -1; *p.err = DYBIT_ERR_INVALID_ARG; }
        }
        return __builtin_amdgcn_readfirstlane(id);
    };
    auto place_of = [&](int id, int token) {
        return (((int64_t)max(id, 0) * p.kv_heads + head) << p.page_shift) + (token & ((1 << p.page_shift) - 1));
    };
    int kid = -1, vid[2] = {-1, -1};                     // pages of the next step's blocks that this wave decodes
    auto look = [&](int step) {
        const int token = lo + step * kStep;
        kid = page_of(token + 16 * wave);
        vid[0] = page_of(token + 32 * vchunk);
        vid[1] = page_of(token + 32 * vchunk + 16);
    };
    auto fetch = [&](Share<D> &s, int step) {
        const int token = lo + step * kStep;
        const int64_t kp = place_of(kid, token + 16 * wave);
        const int left = hi - token - 16 * wave;
        s.valid = kid < 0 ? 0 : left < 16 ? left : 16;
        load_words<D * KB / 32>(p.k_codes + kp * (D * KB / 8) + (lane & 15) * (D * KB / 8) + g4 * (D * KB / 32), s.k);
        s.scale = 0.0f;
        if ((lane & 15) < s.valid && lane < 32) s.scale = (lane < 16 ? p.k_scales : p.v_scales)[kp + (lane & 15)];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t vp = place_of(vid[b], token + 32 * vchunk + 16 * b);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_words<Share<D>::VBYTES>(p.v_codes + (vp + 4 * g4 + i) * (D * VB / 8) + (lane & 15) * (D * VB / 128) + vhalf * Share<D>::VBYTES, s.v[4 * b + i]);
        }
    };
    auto decode = [&](const Share<D> &s, int buffer) {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) lds.k[buffer][wave][j][lane] = key_operand<KB>(s.k, j);
        const Values<VB, D / 32> values(s.v);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) lds.v[buffer][vchunk][vhalf * (D / 32) + j][lane] = values.dim(j);
        if (lane < 16) lds.sk[buffer][16 * wave + lane] = s.scale;
        else if (lane < 32) lds.sv[buffer][16 * wave + lane - 16] = s.scale;
        if (lane == 0) lds.valid[buffer][wave] = s.valid;
    };
    float vref = kFirstRef, vup = kLargeP / kFirstRef;
    auto go = [&](int step, int buffer) {
        const int token = lo + step * kStep;
        f32x4 s[NT][kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                const f16x8 a = lds.k[buffer][b][j][lane];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < TERMS; ++e) s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, r[t].q[e][j], s[t][b], 0, 0, 0);
            }
        }
        float sv[4 * kBlocks], sk[4 * kBlocks], top = 0.0f;
        int valid[kBlocks];
        bool whole = token + kStep <= least;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(&lds.sv[buffer][16 * b + 4 * g4]), y = *reinterpret_cast<const f32x4 *>(&lds.sk[buffer][16 * b + 4 * g4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sv[4 * b + i] = x[i];
                sk[4 * b + i] = y[i];
                top = fmaxf(top, x[i]);
            }
            valid[b] = lds.valid[buffer][b];
            whole = whole && __builtin_amdgcn_readfirstlane(valid[b]) == 16;
        }
        top = max_over_groups(top);
        float shrink = 1.0f;
        if (__builtin_amdgcn_readfirstlane(__float_as_uint(top)) > __float_as_uint(vref)) {
            u32 e = (__float_as_uint(top) >> 23) + 1u;
            e = e > 240u ? 240u : e;
            const float ref = __uint_as_float(__builtin_amdgcn_readfirstlane(e) << 23);
            shrink = vref / ref;
            vref = ref;
            vup = kLargeP / ref;
        }
#pragma unroll
        for (int i = 0; i < 4 * kBlocks; ++i) sv[i] *= vup;
        f16x8 prob[NT][2][TERMS];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float x[4 * kBlocks], mx = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 4 * kBlocks; ++i) {
                x[i] = s[t][i >> 2][i & 3] * (sk[i] * r[t].factor);
                if (!whole) {
                    const int at = 4 * g4 + (i & 3);
                    x[i] = at < valid[i >> 2] && token + 16 * (i >> 2) + at < r[t].seen ? x[i] : -__builtin_inff();
                }
                mx = fmaxf(mx, x[i]);
            }
            const float m = fmaxf(st[t].m, max_over_groups(mx));
            const float base = m == -__builtin_inff() ? 0.0f : m;
            const float keep = __builtin_amdgcn_exp2f(st[t].m - base);
            st[t].m = m;
            if (__any(keep * shrink != 1.0f)) {
                st[t].l *= keep;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) st[t].o[j] *= keep * shrink;
            }
#pragma unroll
            for (int i = 0; i < 4 * kBlocks; ++i) {
                x[i] = __builtin_amdgcn_exp2f(x[i] - base);
                st[t].l += x[i];
                x[i] *= sv[i];
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                u32 w[TERMS][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (TERMS == 2) split_pair(x[8 * c + 2 * i], x[8 * c + 2 * i + 1], w[0][i], w[1][i]);
                    else w[0][i] = round_pair(x[8 * c + 2 * i], x[8 * c + 2 * i + 1]);
                }
#pragma unroll
                for (int e = 0; e < TERMS; ++e) prob[t][c][e] = operand(w[e][0], w[e][1], w[e][2], w[e][3]);
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const f16x8 a = lds.v[buffer][c][j][lane];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < TERMS; ++e) st[t].o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, prob[t][c][e], st[t].o[j], 0, 0, 0);
            }
    };
    Share<D> share;
    if (steps > 0) {
        look(0);
        fetch(share, 0);
        look(1);
        decode(share, 0);
    }
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        const bool more = step + 1 < steps;
        if (more) {
            fetch(share, step + 1);
            look(step + 2);
        }
        go(step, step & (BUFFERS - 1));
        if (BUFFERS == 1) __syncthreads();
        if (more) decode(share, (step + 1) & (BUFFERS - 1));
        __syncthreads();
    }

    const float back = vref / kLargeP * fold<VB>();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (r[t].row < 0) continue;                      // lanes of a row are all here or all not: their sums go over lanes 16 and 32 apart
        st[t].l += __shfl_xor(st[t].l, 16);
        st[t].l += __shfl_xor(st[t].l, 32);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) st[t].o[j] *= back;
        write_row<D>(p, r[t].row, slot, g4, st[t]);
    }
}

template <int D>
void launch_d(const Phase &p, const Plan &plan, int terms, int64_t segments, hipStream_t st)
{
    const dim3 grid((unsigned)(segments * p.kv_heads), (unsigned)plan.row_tiles, (unsigned)plan.slots), block(kThreads);
    if (terms == 1) hipLaunchKernelGGL((attention_wide_kernel<D, 1>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((attention_wide_kernel<D, 2>), grid, block, 0, st, p);
}

}  // namespace

#if DYBIT_KV_K == 8 && DYBIT_KV_V == 8
#define DYBIT_KV_LAUNCH launch_wide_k8v8
#elif DYBIT_KV_K == 8
#define DYBIT_KV_LAUNCH launch_wide_k8v4
#elif DYBIT_KV_V == 8
#define DYBIT_KV_LAUNCH launch_wide_k4v8
#else
#define DYBIT_KV_LAUNCH launch_wide_k4v4
#endif
void DYBIT_KV_LAUNCH(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st)
{
    if (D == 64) launch_d<64>(p, plan, terms, segments, st);
    else if (D == 128) launch_d<128>(p, plan, terms, segments, st);
    else launch_d<256>(p, plan, terms, segments, st);
}

}  // namespace kv
}  // namespace dybit
