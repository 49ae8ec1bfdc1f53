// The key/value cache of codes (dybit_kv_cache): host-side checks and the arithmetic of its layout.
#pragma once
#include "heads.h"

namespace dybit {
namespace kv {

inline dybit_status check(const dybit_kv_cache &c)
{
    for (const dybit_fmt f : {c.k_fmt, c.v_fmt}) {
        const dybit_status st = check_fmt(f);
        if (st != DYBIT_OK) return st;
        if (!f.is_signed || (f.bits != 4 && f.bits != 8)) return DYBIT_ERR_UNSUPPORTED_BITS;
    }
    if (c.heads < 1 || c.heads > 65535 || c.layers < 0 || c.pages < 0 || c.pages > 0x7fffffff) return DYBIT_ERR_INVALID_ARG;
    if (c.head_dim != 64 && c.head_dim != 128 && c.head_dim != 256) return DYBIT_ERR_INVALID_ARG;
    if (c.page_tokens < 16 || c.page_tokens > 1024 || (c.page_tokens & (c.page_tokens - 1))) return DYBIT_ERR_INVALID_ARG;
    if (c.layers && c.pages) {
        for (const void *p : {(const void *)c.k_codes, (const void *)c.k_scales, (const void *)c.v_codes, (const void *)c.v_scales}) {
            if (!p) return DYBIT_ERR_NULL;
            if (!aligned16(p)) return DYBIT_ERR_ALIGNMENT;
        }
    }
    return DYBIT_OK;
}

inline int log2_of(int n)
{
    int s = 0;
    while ((1 << s) < n) ++s;
    return s;
}

}  // namespace kv
}  // namespace dybit
