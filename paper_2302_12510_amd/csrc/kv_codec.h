// Codes of the cache to operands of v_mfma_f32_16x16x32_f16, in registers.
//
// Keys: a lane holds a run of one token's codes and takes eight at a time, in their order.  Values: a lane holds the same dims of
// eight tokens and takes one dim of all of them at a time.  8-bit codes come out 2^-14-fold (as in dybit_codec.h, whose identity for
// the value of a code is used), which the caller multiplies back into the accumulators.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dybit {
namespace kv {

typedef uint32_t u32;
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));

template <int BITS> constexpr float fold() { return BITS == 8 ? 16384.0f : 1.0f; }

// x: two 8-bit codes, each in both bytes of its half: the sign is the half's own sign bit then.  c, the low seven bits, is the
// subnormal half c 2^-24, so one fma makes n = 2^7 - c on a scale of 2^-9 of it, whose bit pattern counts down as the code's value
// counts up (dybit_codec.h): 13 exponents less the pattern is the value, 2^-14-fold.  Five instructions a pair with the
// byte permute before it.
__device__ __forceinline__ u32 halves_of_doubled(u32 x)
{
    const f16x2 c = __builtin_bit_cast(f16x2, x & 0x007f007fu);
    const f16x2 n = __builtin_elementwise_fma(c, (f16x2){(_Float16)-32768.0f, (_Float16)-32768.0f}, (f16x2){(_Float16)0.25f, (_Float16)0.25f});
    const u32 v = __builtin_bit_cast(u32, __builtin_bit_cast(u16x2, 0x34003400u) - __builtin_bit_cast(u16x2, n));
    return v | (x & 0x80008000u);
}

// Eight 4-bit codes of a word -> high bytes of their halves (the low bytes are zero): even codes, odd codes.
__device__ __forceinline__ void high_bytes(u32 w, u32 &even, u32 &odd)
{
    const u32 tlo = 0x3A383400u, thi = 0x44403E3Cu;                                       // of 0, .25, .5, .75, 1, 1.5, 2, 4
    even = __builtin_amdgcn_perm(thi, tlo, w & 0x07070707u) | ((w << 4) & 0x80808080u);
    odd = __builtin_amdgcn_perm(thi, tlo, (w >> 4) & 0x07070707u) | (w & 0x80808080u);
}

__device__ __forceinline__ f16x8 operand(u32 a, u32 b, u32 c, u32 d)
{
    return __builtin_bit_cast(f16x8, u32x4{a, b, c, d});
}

// Eight consecutive codes of a key, group j of the run in w.
template <int BITS>
__device__ __forceinline__ f16x8 key_operand(const u32 *w, int j)
{
    if constexpr (BITS == 8) {
        const u32 a = w[2 * j], b = w[2 * j + 1];
        return operand(halves_of_doubled(__builtin_amdgcn_perm(a, a, 0x01010000u)), halves_of_doubled(__builtin_amdgcn_perm(a, a, 0x03030202u)),
                       halves_of_doubled(__builtin_amdgcn_perm(b, b, 0x01010000u)), halves_of_doubled(__builtin_amdgcn_perm(b, b, 0x03030202u)));
    } else {
        u32 e, o;
        high_bytes(w[j], e, o);
        return operand(__builtin_amdgcn_perm(o, e, 0x040c000cu), __builtin_amdgcn_perm(o, e, 0x050c010cu),
                       __builtin_amdgcn_perm(o, e, 0x060c020cu), __builtin_amdgcn_perm(o, e, 0x070c030cu));
    }
}

// Values of eight tokens, DIMS dims each: words w[token][..].  prepare() once, then operand j = dim j of all eight.
template <int BITS, int DIMS> struct Values;
template <int DIMS> struct Values<8, DIMS> {
    static constexpr int WORDS = (DIMS + 3) / 4;
    const u32 (*w)[WORDS];
    __device__ __forceinline__ explicit Values(const u32 (*words)[WORDS]) : w(words) {}
    __device__ __forceinline__ u32 pair(int a, int j) const
    {
        const u32 k = j & 3;
        return halves_of_doubled(__builtin_amdgcn_perm(w[a + 1][j >> 2], w[a][j >> 2], k | k << 8 | (k + 4) << 16 | (k + 4) << 24));
    }
    __device__ __forceinline__ f16x8 dim(int j) const { return operand(pair(0, j), pair(2, j), pair(4, j), pair(6, j)); }
};
template <int DIMS> struct Values<4, DIMS> {
    static constexpr int WORDS = (DIMS + 7) / 8;
    static constexpr bool JOINED = DIMS <= 4;                           // two tokens' codes in one word
    u32 e[JOINED ? 4 : 8][WORDS], o[JOINED ? 4 : 8][WORDS];
    __device__ __forceinline__ explicit Values(const u32 (*w)[WORDS])
    {
        if constexpr (JOINED) {
#pragma unroll
            for (int t = 0; t < 4; ++t) high_bytes(w[2 * t][0] | w[2 * t + 1][0] << 16, e[t][0], o[t][0]);
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int i = 0; i < WORDS; ++i) high_bytes(w[t][i], e[t][i], o[t][i]);
        }
    }
    __device__ __forceinline__ u32 pair(int a, int j) const
    {
        const u32 k = (j & 7) >> 1;
        if constexpr (JOINED) {
            const u32 x = j & 1 ? o[a / 2][0] : e[a / 2][0];
            return __builtin_amdgcn_perm(0u, x, 0x000c000cu | k << 8 | (k + 2) << 24);
        } else {
            const u32 x = j & 1 ? o[a][j >> 3] : e[a][j >> 3], y = j & 1 ? o[a + 1][j >> 3] : e[a + 1][j >> 3];
            return __builtin_amdgcn_perm(y, x, 0x000c000cu | k << 8 | (k + 4) << 24);
        }
    }
    __device__ __forceinline__ f16x8 dim(int j) const { return operand(pair(0, j), pair(2, j), pair(4, j), pair(6, j)); }
};

// Two floats rounded to halves, and what that leaves of them.  The rounded pair is taken for what it is once: left to itself the compiler
// rounds a product to fp16 here in one step and there in two, and the rest would belong to another half than the one that is used.
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32 round_pair(float a, float b) { return __builtin_bit_cast(u32, __builtin_convertvector((f32x2{a, b}), f16x2)); }
__device__ __forceinline__ void split_pair(float a, float b, u32 &high, u32 &low, float times = 1.0f)
{
    high = round_pair(a, b);
    asm("" : "+v"(high));
    const f16x2 h = __builtin_bit_cast(f16x2, high);
    low = round_pair((a - (float)h[0]) * times, (b - (float)h[1]) * times);
}

// The rest of a split probability is taken 2^10-fold, and the values for its first half too (exact: they are within 2^-20 and 2^12
// then), so that the rests of small probabilities are not lost below the smallest half.
constexpr float kRest = 1024.0f;
__device__ __forceinline__ f16x8 times_rest(f16x8 a) { return a * (f16x8)((_Float16)kRest); }

// BYTES (1, 2, 4, 8, 16, 32, 64) from p into whole words.
template <int BYTES>
__device__ __forceinline__ void load_words(const uint8_t *p, u32 *w)
{
    if constexpr (BYTES == 1) w[0] = *p;
    else if constexpr (BYTES == 2) w[0] = *reinterpret_cast<const unsigned short *>(p);
    else if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const u32 *>(p);
    else if constexpr (BYTES == 8) {
        const u32x2 r = *reinterpret_cast<const u32x2 *>(p);
        w[0] = r.x; w[1] = r.y;
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const u32x4 r = *reinterpret_cast<const u32x4 *>(p + 16 * i);
            w[4 * i] = r.x; w[4 * i + 1] = r.y; w[4 * i + 2] = r.z; w[4 * i + 3] = r.w;
        }
    }
}

// The largest of a value over the four groups of 16 lanes.
__device__ __forceinline__ float max_over_groups(float x)
{
    const u32 b = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const u32 y = __float_as_uint(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
    const auto s = __builtin_amdgcn_permlane16_swap(y, y, false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// The largest of a value over a lane's row of 16.
__device__ __forceinline__ float max_over_row(float x)
{
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, true)));   // row_ror:8
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xf, 0xf, true)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x122, 0xf, 0xf, true)));
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x121, 0xf, 0xf, true)));
}

}  // namespace kv
}  // namespace dybit
