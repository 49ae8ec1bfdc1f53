// RMS norm of every query and key head with the rotation by the token's position, in one pass, and its gradient.
//
// A head is a list of D / 2 pairs: the rotated ones, then neighbours that pass unturned.  A lane
// holds V consecutive pairs, 2 V elements in two vector accesses, so a rotation never leaves its lane; the lanes of a head share
// only the sum of squares (and, backward, the sum of h x).  A wave takes the heads of one token side by side: its rows of the
// cosine and sine tables, and the weights, are read once for all of them.
//   forward   n = x r w,  r = 1 / sqrt(mean x^2 + eps),  y = R n
//   backward  g' = R^T g,  h = g' w,  dx = r (h - x r^2 mean(h x)),  dw = sum g' x r
// Both are bound by memory: a head is read and written once (backward: inputs and gradients read, written once).  8191 tokens of 40
// heads of 128 in bf16, 171 MB: 34.0 to 39.5 us over cards, 4.3 to 5.0 TB/s, where a device copy of as much takes 33; a training step of
// 4097 tokens of 32 heads of 64 in fp32: 14 us forward, 22 us for its 101 MB backward, 4.6 to add the weights' partial gradients up.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "heads.h"

namespace dybit {
namespace headnorm {

using heads::Loose;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostBlocks = 1024;                 // of the backward pass, whose partial sums of the weights' gradients are one row a block

struct Args {
    const void *x[2];                             // queries, keys
    const void *g[2];
    void *y[2];
    const float *w[2];
    int64_t xt[2], xh[2], gt[2], gh[2], yt[2], yh[2];       // strides by token and by head
    int32_t heads[2];
    const int64_t *positions;
    const float *cos, *sin;
    int64_t table_rows, tokens;
    int32_t D, half;                              // half: rotated pairs
    int32_t neighbours, parts, lanes_log2;        // parts: waves per token; lanes per head, a power of two
    int32_t turned, runs;                         // runs of V pairs of a head: the rotated ones, all of them
    float eps;
    int *err;
    float *partial;                               // [blocks][2][D]
};

// Runs of V pairs that cover a head, rotated pairs and the others apart.  Where V does not divide either number, its last run starts early:
// the first `skip` pairs of it are the run's before as well, count once in the sums, and are stored twice, with one value (4000 tokens, 40
// heads of 128 in fp16, 35 pairs of them rotated: 40 us, with pairs one by one 79).
template <int V>
struct Run {
    int pair, skip;
    __device__ __forceinline__ Run(const Args &p, int n)
    {
        const int from = n < p.turned ? 0 : p.half, all = n < p.turned ? p.half : p.D / 2 - p.half, at = (n < p.turned ? n : n - p.turned) * V;
        const int first = min(at, all - V);
        pair = n < p.runs ? from + first : p.D / 2;
        skip = at - first;
    }
};

// Where the V pairs from p on lie: their first and their second elements as two runs, or interleaved in one run of 2 V.
template <int V>
struct Place {
    int first, second;
    bool woven;
    __device__ __forceinline__ Place(int p, int half, int neighbours)
    {
        woven = neighbours || p >= half;
        first = woven ? 2 * p : p;
        second = woven ? 2 * p + V : p + half;
    }
};

template <class T, int V>
__device__ __forceinline__ void load_pairs(const T *row, const Place<V> &at, float (&a)[V], float (&b)[V])
{
    float u[V], v[V];
    Loose<T, V>::load(row + at.first, u);
    Loose<T, V>::load(row + at.second, v);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float s = 2 * i < V ? u[(2 * i) % V] : v[(2 * i) % V], t = 2 * i + 1 < V ? u[(2 * i + 1) % V] : v[(2 * i + 1) % V];
        a[i] = at.woven ? s : u[i];
        b[i] = at.woven ? t : v[i];
    }
}

template <class T, int V>
__device__ __forceinline__ void store_pairs(T *row, const Place<V> &at, const float (&a)[V], const float (&b)[V])
{
    float u[V], v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float s = i % 2 ? b[i / 2] : a[i / 2], t = (V + i) % 2 ? b[(V + i) / 2] : a[(V + i) / 2];
        u[i] = at.woven ? s : a[i];
        v[i] = at.woven ? t : b[i];
    }
    Loose<T, V>::store(row + at.first, u);
    Loose<T, V>::store(row + at.second, v);
}

// Over a head's lanes (a power of two): lanes of a row of 16 by data-parallel permutes, rows by the rows' exchange.
template <int PERMUTE>
__device__ __forceinline__ float add_permuted(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), PERMUTE, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_over(float x, int lanes)
{
    if (lanes > 1) x = add_permuted<0xB1>(x);              // quad_perm [1,0,3,2]
    if (lanes > 2) x = add_permuted<0x4E>(x);              // quad_perm [2,3,0,1]
    if (lanes > 4) x = add_permuted<0x141>(x);             // row_half_mirror
    if (lanes > 8) x = add_permuted<0x140>(x);             // row_mirror
    if (lanes > 16) x += __shfl_xor(x, 16);
    if (lanes > 32) x += __shfl_xor(x, 32);
    return x;
}

// A pair by its angle, or as it is (an infinite element behind the rotated ones is none of its neighbour's business).
__device__ __forceinline__ void turn(float &a, float &b, float c, float s, bool turns)
{
    const float u = a * c - b * s, v = b * c + a * s;
    a = turns ? u : a;
    b = turns ? v : b;
}

// K: groups of V pairs per lane (1 except for heads that are wider than 64 lanes hold).
// OVER: some runs overlap (a variant of its own: the others would lose 2 % to it).
template <class T, int V, int K, bool BACK, bool OVER>
__global__ __launch_bounds__(kThreads) void head_norm_kernel(const Args p)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lanes = 1 << p.lanes_log2, group = lane >> p.lanes_log2, groups = 64 >> p.lanes_log2, at = lane & (lanes - 1);
    int pair[K], skip[K];
    bool turns[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        pair[k] = (at + k * lanes) * V;
        skip[k] = 0;
        if constexpr (OVER) {
            const Run<V> run(p, at);
            pair[k] = run.pair;
            skip[k] = run.skip;
        }
        turns[k] = pair[k] < p.half;
    }
    float dw[2][K][2 * V];
    if (BACK) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) dw[a][k][i] = 0.0f;
    }
    const int64_t units = p.tokens * p.parts;
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units; unit += (int64_t)gridDim.x * kWaves) {
        const int64_t t = unit / p.parts;
        const int part = (int)(unit - t * p.parts);
        const int64_t position = p.positions[t];
        const bool known = position >= 0 && position < p.table_rows;
        float c[K][V], s[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < V; ++i) { c[k][i] = 1.0f; s[k][i] = 0.0f; }
            if (known && turns[k]) {
                Loose<float, V>::load(p.cos + position * p.half + pair[k], c[k]);
                Loose<float, V>::load(p.sin + position * p.half + pair[k], s[k]);
            }
        }
        if (!known && lane == 0) *p.err = DYBIT_ERR_INVALID_ARG;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            float wa[K][V], wb[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (p.heads[a] && pair[k] < p.D / 2) load_pairs<float, V>(p.w[a], Place<V>(pair[k], p.half, p.neighbours), wa[k], wb[k]);
            // the waves of a token and the groups of a wave take turns at the heads; all lanes stay for the sums
            for (int first = part * groups; first < p.heads[a]; first += p.parts * groups) {
                const int h = first + group;
                const bool in = h < p.heads[a];
                float xa[K][V], xb[K][V], ga[K][V], gb[K][V];
                float squares = 0.0f, dot = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (in && pair[k] < p.D / 2) {
                        const Place<V> place(pair[k], p.half, p.neighbours);
                        load_pairs<T, V>((const T *)p.x[a] + t * p.xt[a] + h * p.xh[a], place, xa[k], xb[k]);
                        if (BACK) load_pairs<T, V>((const T *)p.g[a] + t * p.gt[a] + h * p.gh[a], place, ga[k], gb[k]);
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            squares += xa[k][i] * xa[k][i] + xb[k][i] * xb[k][i];
                            if (BACK) {
                                turn(ga[k][i], gb[k][i], c[k][i], -s[k][i], turns[k]);
                                dot += ga[k][i] * wa[k][i] * xa[k][i] + gb[k][i] * wb[k][i] * xb[k][i];
                            }
                        }
                        if (OVER && skip[k]) {                        // K is 1: the sums are this run's alone
                            squares = dot = 0.0f;
#pragma unroll
                            for (int i = 1; i < V; ++i) {
                                if (i < skip[k]) continue;
                                squares += xa[k][i] * xa[k][i] + xb[k][i] * xb[k][i];
                                if (BACK) dot += ga[k][i] * wa[k][i] * xa[k][i] + gb[k][i] * wb[k][i] * xb[k][i];
                            }
                        }
                    }
                }
                squares = sum_over(squares, lanes);
                if (BACK) dot = sum_over(dot, lanes);
                const float r = known ? 1.0f / __builtin_sqrtf(squares / (float)p.D + p.eps) : __builtin_nanf("");
                const float pull = BACK ? dot / (float)p.D * r * r : 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (!in || pair[k] >= p.D / 2) continue;
                    float ya[V], yb[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        if (BACK) {
                            ya[i] = r * (ga[k][i] * wa[k][i] - xa[k][i] * pull);
                            yb[i] = r * (gb[k][i] * wb[k][i] - xb[k][i] * pull);
                            if (known) {
                                dw[a][k][i] += ga[k][i] * (xa[k][i] * r);
                                dw[a][k][V + i] += gb[k][i] * (xb[k][i] * r);
                            }
                        } else {
                            ya[i] = xa[k][i] * r * wa[k][i];
                            yb[i] = xb[k][i] * r * wb[k][i];
                            turn(ya[i], yb[i], c[k][i], s[k][i], turns[k]);
                        }
                    }
                    store_pairs<T, V>((T *)p.y[a] + t * p.yt[a] + h * p.yh[a], Place<V>(pair[k], p.half, p.neighbours), ya, yb);
                }
            }
        }
    }
    if constexpr (!BACK) return;
    // the weights' gradients: over the groups of a wave, then over its block's waves, into the block's row
    __shared__ float sums[kWaves][2][512];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) {
                float x = dw[a][k][i];
                for (int off = lanes; off < 64; off <<= 1) x += __shfl_xor(x, off);
                dw[a][k][i] = x;
            }
            if (group == 0 && pair[k] < p.D / 2) {
                const Place<V> place(pair[k], p.half, p.neighbours);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    sums[wave][a][place.woven ? 2 * (pair[k] + i) : place.first + i] = dw[a][k][i];
                    sums[wave][a][place.woven ? 2 * (pair[k] + i) + 1 : place.second + i] = dw[a][k][V + i];
                }
            }
        }
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * p.D; j += kThreads) {
        const int a = j >= p.D, d = j - a * p.D;
        float x = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += sums[w][a][d];
        p.partial[(int64_t)blockIdx.x * 2 * p.D + j] = x;
    }
}

// Sums the blocks' rows: a workgroup per 16 columns, 64 rows at a time, in an order that the number of blocks fixes.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void head_norm_sum_kernel(const float *partial, int blocks, int D, float *dwq, float *dwk)
{
    constexpr int ROWS = kSumThreads / 16, TURNS = kMostBlocks / ROWS;
    const int at = threadIdx.x & 15, column = blockIdx.x * 16 + at, row = threadIdx.x >> 4;
    float x = 0.0f;
    if (column < 2 * D) {
        float y[TURNS];                                    // all requested before the first is added
#pragma unroll
        for (int k = 0; k < TURNS; ++k) y[k] = row + k * ROWS < blocks ? partial[(int64_t)(row + k * ROWS) * 2 * D + column] : 0.0f;
#pragma unroll
        for (int k = 0; k < TURNS; ++k) x += y[k];
    }
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    __shared__ float sums[kSumThreads / 64][16];
    if ((threadIdx.x & 63) < 16) sums[threadIdx.x >> 6][at] = x;
    __syncthreads();
    if (threadIdx.x >= 16 || column >= 2 * D) return;
    x = 0.0f;
#pragma unroll
    for (int w = 0; w < kSumThreads / 64; ++w) x += sums[w][at];
    if (column < D) dwq[column] = x;
    else if (dwk) dwk[column - D] = x;
}

// Waves of a token backward: two keep kMostBlocks' waves in work from 2048 tokens on; fewer tokens are shared out more finely, down to one
// head a wave and turn.
int64_t backward_parts(int64_t tokens, int64_t turns)
{
    const int64_t wanted = std::max<int64_t>(2, kMostBlocks * kWaves / std::max<int64_t>(1, tokens));
    return std::max<int64_t>(1, std::min(turns, wanted));
}
int blocks_of(int64_t tokens, int64_t parts) { return (int)std::min<int64_t>(kMostBlocks, (tokens * parts + kWaves - 1) / kWaves); }

// Waves of a token forward: about kForward in all, each with as many turns at the heads as the others.  More of them pay their start and
// the token's row of the tables again, fewer leave the device idle (40 heads of 128 in bf16, us: 4096 tokens one wave a token 15.6, two
// 16.5; 3000 tokens one 12.4, two 13.2, four 15.5; 1500 tokens one 9.6, two 8.7, four 10.0).
constexpr int64_t kForward = 4096;
int forward_parts(int64_t tokens, int turns)
{
    const int wanted = (int)std::min<int64_t>(turns, std::max<int64_t>(1, (kForward + tokens / 2) / std::max<int64_t>(1, tokens)));
    const int rounds = (turns + wanted - 1) / wanted;
    return (turns + rounds - 1) / rounds;
}

template <class T, bool BACK>
int launch(Args &p, int V, hipStream_t st)
{
    int blocks;
    p.turned = (p.half + V - 1) / V;
    p.runs = p.turned + (p.D / 2 - p.half + V - 1) / V;
    const bool over = p.half % V || p.D / 2 % V;
    while (p.lanes_log2 < 6 && 1 << p.lanes_log2 < p.runs) ++p.lanes_log2;
    const int groups = 64 >> p.lanes_log2, turns = (p.heads[0] + groups - 1) / groups;
    if (BACK) {
        p.parts = (int)backward_parts(p.tokens, turns);
        blocks = blocks_of(p.tokens, p.parts);
    } else {
        p.parts = forward_parts(p.tokens, std::max(1, turns));
        blocks = (int)((p.tokens * p.parts + kWaves - 1) / kWaves);
    }
    if (p.parts < 1) p.parts = 1;
    const dim3 grid((unsigned)blocks), block(kThreads);
#define DYBIT_HN(V, K) \
    if (over && V > 1) hipLaunchKernelGGL((head_norm_kernel<T, V, K, BACK, (V > 1)>), grid, block, 0, st, p); \
    else hipLaunchKernelGGL((head_norm_kernel<T, V, K, BACK, false>), grid, block, 0, st, p)
    if constexpr (sizeof(T) == 2 && !BACK)
        if (V == 8) { DYBIT_HN(8, 1); return blocks; }
    if (V == 4) { DYBIT_HN(4, 1); }
    else if (V == 2) { DYBIT_HN(2, 1); }
    else { DYBIT_HN(1, 4); }
#undef DYBIT_HN
    return blocks;
}

dybit_status run(bool back, const dybit_heads *g, const dybit_heads *x, const dybit_heads *y, const float *const *w, const int64_t *positions,
                 const float *cos_table, const float *sin_table, int64_t table_rows, int32_t rotary, int32_t neighbours, float eps,
                 float *const *dw, float *workspace, hipStream_t st)
{
    const bool keys = x[1].heads > 0;
    Args p{};
    for (int a = 0; a < (keys ? 2 : 1); ++a)
        for (const dybit_heads *h : {x + a, y + a, g ? g + a : x + a}) {
            const dybit_status s = heads::check(*h);
            if (s != DYBIT_OK) return s;
            if (!heads::same_shape(*h, x[a]) || h->tokens != x[0].tokens || h->head_dim != x[0].head_dim || h->type != x[0].type)
                return DYBIT_ERR_INVALID_ARG;
            if (!w[a]) return DYBIT_ERR_NULL;
        }
    if (!keys && (y[1].heads || (g && g[1].heads))) return DYBIT_ERR_INVALID_ARG;
    const int D = x[0].head_dim;
    if (D % 2 || D > 512 || rotary < 2 || rotary % 2 || rotary > D || table_rows < 0 || !(eps >= 0.0f) || (neighbours != 0 && neighbours != 1))
        return DYBIT_ERR_INVALID_ARG;
    if (back && (!dw[0] || (keys && !dw[1]) || !workspace)) return DYBIT_ERR_NULL;
    if (back && !aligned16(workspace)) return DYBIT_ERR_ALIGNMENT;
    if (x[0].tokens == 0 && !back) return DYBIT_OK;
    if (x[0].tokens && (!positions || !cos_table || !sin_table)) return DYBIT_ERR_NULL;
    // pairs of a lane: 16-byte accesses, but backward four pairs, whose registers leave room for four waves a SIMD (4096 tokens, 40 heads of
    // 128 in bf16, both passes: eight pairs 66 us, four 51)
    int V = x[0].type == DYBIT_F32 || back ? 4 : 8;
    auto fits = [&](int v) {
        const int turned = rotary / 2, rest = D / 2 - turned;
        return turned >= v && (rest == 0 || rest >= v) && (turned + v - 1) / v + (rest + v - 1) / v <= 64;
    };
    while (V > 1 && !fits(V)) V /= 2;
    for (int a = 0; a < (keys ? 2 : 1); ++a) {
        p.x[a] = x[a].data; p.xt[a] = x[a].token_stride; p.xh[a] = x[a].head_stride;
        p.y[a] = y[a].data; p.yt[a] = y[a].token_stride; p.yh[a] = y[a].head_stride;
        if (g) { p.g[a] = g[a].data; p.gt[a] = g[a].token_stride; p.gh[a] = g[a].head_stride; }
        p.w[a] = w[a];
        p.heads[a] = x[a].heads;
    }
    p.positions = positions; p.cos = cos_table; p.sin = sin_table; p.table_rows = table_rows; p.tokens = x[0].tokens;
    p.D = D; p.half = rotary / 2; p.neighbours = neighbours; p.eps = eps; p.partial = workspace;
    p.err = async_error_word();
    if (!p.err) return DYBIT_ERR_HIP;
    int blocks = 0;
    if (p.tokens) {
        switch (x[0].type) {
            case DYBIT_F32: blocks = back ? launch<float, true>(p, V, st) : launch<float, false>(p, V, st); break;
            case DYBIT_F16: blocks = back ? launch<_Float16, true>(p, V, st) : launch<_Float16, false>(p, V, st); break;
            default: blocks = back ? launch<__bf16, true>(p, V, st) : launch<__bf16, false>(p, V, st); break;
        }
    }
    if (back)
        hipLaunchKernelGGL(head_norm_sum_kernel, dim3((unsigned)((2 * D + 15) / 16)), dim3(kSumThreads), 0, st, workspace, blocks,
                           D, dw[0], keys ? dw[1] : nullptr);
    return launch_status();
}

}  // namespace headnorm
}  // namespace dybit

extern "C" dybit_status dybit_head_norm_rope(dybit_heads q, dybit_heads k, const float *q_weight, const float *k_weight,
                                             const int64_t *positions, const float *cos_table, const float *sin_table, int64_t table_rows,
                                             int32_t rotary, int32_t neighbours, float eps, dybit_heads q_out, dybit_heads k_out,
                                             dybit_stream stream)
{
    const dybit_heads x[2] = {q, k}, y[2] = {q_out, k_out};
    const float *w[2] = {q_weight, k_weight};
    return dybit::headnorm::run(false, nullptr, x, y, w, positions, cos_table, sin_table, table_rows, rotary, neighbours, eps, nullptr, nullptr,
                                 (hipStream_t)stream);
}

extern "C" size_t dybit_head_norm_rope_bwd_workspace(int64_t tokens, int32_t heads, int32_t head_dim)
{
    if (tokens < 0 || heads < 0 || head_dim < 1) return 0;
    // turns at the heads depend on the alignment of the call's tensors: at most one a head
    const int64_t parts = dybit::headnorm::backward_parts(tokens, heads);
    return (size_t)(tokens ? dybit::headnorm::blocks_of(tokens, parts) : 1) * 2 * (size_t)head_dim;
}

extern "C" dybit_status dybit_head_norm_rope_bwd(dybit_heads grad_q, dybit_heads grad_k, dybit_heads q, dybit_heads k,
                                                 const float *q_weight, const float *k_weight, const int64_t *positions,
                                                 const float *cos_table, const float *sin_table, int64_t table_rows,
                                                 int32_t rotary, int32_t neighbours, float eps, dybit_heads dq, dybit_heads dk,
                                                 float *q_weight_grad, float *k_weight_grad, float *workspace, dybit_stream stream)
{
    const dybit_heads g[2] = {grad_q, grad_k}, x[2] = {q, k}, y[2] = {dq, dk};
    const float *w[2] = {q_weight, k_weight};
    float *dw[2] = {q_weight_grad, k_weight_grad};
    return dybit::headnorm::run(true, g, x, y, w, positions, cos_table, sin_table, table_rows, rotary, neighbours, eps, dw, workspace,
                                 (hipStream_t)stream);
}
