// Rows of heads (dybit_heads): element types, vector access, host-side checks.  Shared by the norm with rotation, the cache's
// encoder and the attention.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/dybit.h"
#include "dybit_host.h"

namespace dybit {
namespace heads {

// V consecutive elements as one aligned access, as floats.
template <class T, int V> struct Pack {
    typedef T raw __attribute__((ext_vector_type(V)));
    static __device__ __forceinline__ void load(const T *p, float (&x)[V])
    {
        const raw r = *reinterpret_cast<const raw *>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (float)r[i];
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[V])
    {
        raw r;
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = (T)x[i];               // one rounding, to nearest even
        *reinterpret_cast<raw *>(p) = r;
    }
};
template <class T> struct Pack<T, 1> {
    static __device__ __forceinline__ void load(const T *p, float (&x)[1]) { x[0] = (float)*p; }
    static __device__ __forceinline__ void store(T *p, const float (&x)[1]) { *p = (T)x[0]; }
};

// The same from wherever an element may start: one access too, which the hardware splits where it crosses a line.
template <class T, int V> struct Loose {
    typedef T raw __attribute__((ext_vector_type(V), aligned(alignof(T))));
    static __device__ __forceinline__ void load(const T *p, float (&x)[V])
    {
        const raw r = *reinterpret_cast<const raw *>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (float)r[i];
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[V])
    {
        raw r;
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = (T)x[i];               // one rounding, to nearest even
        *reinterpret_cast<raw *>(p) = r;
    }
};
template <class T> struct Loose<T, 1> : Pack<T, 1> {};

inline int type_bytes(int type) { return type == DYBIT_F32 ? 4 : 2; }

inline dybit_status check(const dybit_heads &h)
{
    if (h.type != DYBIT_F32 && h.type != DYBIT_F16 && h.type != DYBIT_BF16) return DYBIT_ERR_INVALID_ARG;
    if (h.tokens < 0 || h.heads < 0 || h.head_dim < 1 || h.tokens > 0x7fffffff) return DYBIT_ERR_INVALID_ARG;
    if (!h.data && h.tokens && h.heads) return DYBIT_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(h.data) % (unsigned)type_bytes(h.type)) return DYBIT_ERR_ALIGNMENT;
    return DYBIT_OK;
}

inline bool same_shape(const dybit_heads &a, const dybit_heads &b)
{
    return a.tokens == b.tokens && a.heads == b.heads && a.head_dim == b.head_dim && a.type == b.type;
}

// Whether every head starts on a multiple of `elements` elements.
inline bool aligned(const dybit_heads &h, int elements)
{
    return reinterpret_cast<uintptr_t>(h.data) % (unsigned)(elements * type_bytes(h.type)) == 0 &&
           (h.tokens <= 1 || h.token_stride % elements == 0) && (h.heads <= 1 || h.head_stride % elements == 0);
}

}  // namespace heads
}  // namespace dybit
