// Attention over the cache of codes: what its kernels, the choice between them and the join of their parts share.
#pragma once
#include "kv_cache.h"

namespace dybit {
namespace kv {

// One phase of an attention call: queries over the tokens that each segment (a sequence's own pages, or a group's prefix) holds.
struct Phase {
    const void *q;
    void *out;
    int64_t q_token, q_head, out_token, out_head;      // strides
    int32_t type, q_vectors, out_vectors;              // vectors: heads start on multiples of eight elements
    const uint8_t *k_codes, *v_codes;
    const float *k_scales, *v_scales;
    int64_t pages;
    int32_t kv_heads, group, page_shift;               // group: query heads per key head
    const int32_t *tables, *lengths, *starts, *members;// members: first sequence of each group (prefix), or NULL
    int64_t table_width, tokens, sequences;
    int64_t max_queries, cap;                          // cap: most tokens of a segment that are looked at
    int32_t causal, chunk;                             // chunk: tokens of a segment that one workgroup goes through
    float scale;                                       // times log2(e)
    float *part_out, *part_stat;                       // partial results [token][query head][slot][D], (maximum, sum); NULL: write out
    int64_t slot0, slots;                              // first slot of the phase; slots of a row
    int *err;
};

// Query tokens and keys of a segment, clamped to what the call may touch.
struct Segment {
    int64_t first;
    int32_t count, length;
    bool odd;                                          // something was out of range
};

__device__ __forceinline__ Segment segment(const Phase &p, int s)
{
    Segment g;
    int64_t a = s, b = s + 1;
    if (p.members) {
        a = p.members[s];
        b = p.members[s + 1];
        g.odd = a < 0 || b < a || b > p.sequences;
        a = a < 0 ? 0 : a > p.sequences ? p.sequences : a;
        b = b < a ? a : b > p.sequences ? p.sequences : b;
    } else {
        g.odd = false;
    }
    if (p.starts) {
        a = p.starts[a];
        b = p.starts[b];
    }
    g.odd |= a < 0 || b < a || b > p.tokens || b - a > p.max_queries;
    a = a < 0 ? 0 : a > p.tokens ? p.tokens : a;
    b = b < a ? a : b > p.tokens ? p.tokens : b;
    g.first = a;
    g.count = (int32_t)(b - a > p.max_queries ? p.max_queries : b - a);
    int64_t n = p.lengths[s];
    g.odd |= n < 0 || n > p.cap;
    g.length = (int32_t)(n < 0 ? 0 : n > p.cap ? p.cap : n);
    return g;
}

// Keys that query i of a segment sees.
__device__ __forceinline__ int visible(const Phase &p, const Segment &g, int i)
{
    const int n = p.causal ? g.length - (g.count - 1 - i) : g.length;
    return n < 0 ? 0 : n;
}

// How a phase is run: decided on the host from sizes alone.
struct Plan {
    bool wide;                                         // kv_attention_wide.hip, else kv_attention.hip
    int32_t tiles16;                                   // 16-row tiles of a wave of the latter: 1 or 2
    int32_t chunk;
    int64_t row_tiles, slots;
};

void launch_k8v8(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
void launch_k8v4(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
void launch_k4v8(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
void launch_k4v4(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
void launch_wide_k8v8(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
void launch_wide_k8v4(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
void launch_wide_k4v8(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
void launch_wide_k4v4(const Phase &p, const Plan &plan, int D, int terms, int64_t segments, hipStream_t st);
// The wide kernel: rows of a wave, and waves of a workgroup.  Eight waves leave a wave 256 registers; four, 512.
constexpr int kWideRows = 32;
constexpr int wide_waves(int D, int terms) { return D * terms >= 256 ? 4 : 8; }

}  // namespace kv
}  // namespace dybit
