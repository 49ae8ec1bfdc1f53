"""Oracle of the key/value cache: norm with rotation and its gradient, append, attention, copies of pages, in 64 bits
(numpy), written from their definitions.  Bounds on the device's error are computed beside the results, from the number of
roundings that a result goes through."""
from __future__ import annotations

import numpy as np

from . import dybit_ref as R

U = 2.0 ** -24                                            # unit roundoff of fp32
HALF_ULP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}     # of one rounding to the type, relative (bf16: 8 bits)
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -24, "bf16": 2.0 ** -133}       # spacing of its subnormals


def pairs(rotary: int, neighbours: bool):
    i = np.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if neighbours else (i, i + rotary // 2)


def rotate(x, cos, sin, neighbours):
    """x [T][H][D], cos / sin [T][pairs]."""
    a, b = pairs(2 * cos.shape[1], neighbours)
    y = x.copy()
    c, s = cos[:, None], sin[:, None]
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def head_norm_rope(x, w, cos, sin, eps, neighbours, dtype):
    """(y, bound): the sum of squares, its root, the division and the products lose at most 32 roundings of the pair's terms."""
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y = rotate(n, cos, sin, neighbours)
    terms = rotate(np.abs(n), np.abs(cos), -np.abs(sin), neighbours)
    a, b = pairs(2 * cos.shape[1], neighbours)
    terms[..., b] = np.abs(n)[..., b] * np.abs(cos)[:, None] + np.abs(n)[..., a] * np.abs(sin)[:, None]
    return y, 32 * U * terms + HALF_ULP[dtype] * np.abs(y) + TINY[dtype]


def head_norm_rope_bwd(g, x, w, cos, sin, eps, neighbours, dtype):
    """(dx, bound, dw, bound)."""
    D = x.shape[-1]
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    back = rotate(g, cos, -sin, neighbours)
    size = rotate(np.abs(g), np.abs(cos), -np.abs(sin), neighbours)
    a, b = pairs(2 * cos.shape[1], neighbours)
    size[..., b] = np.abs(g)[..., b] * np.abs(cos)[:, None] + np.abs(g)[..., a] * np.abs(sin)[:, None]
    h = back * w
    dx = r * (h - n * (h * n).mean(-1, keepdims=True))
    terms = r * (size * np.abs(w) + np.abs(n) * (size * np.abs(w) * np.abs(n)).mean(-1, keepdims=True))
    dw = (back * n).sum((0, 1))
    # sums over tokens and heads in any order: a rounding for every term at most
    many = x.shape[0] * x.shape[1] + 64
    return dx, 64 * U * terms + HALF_ULP[dtype] * np.abs(dx) + TINY[dtype], dw, many * U * (size * np.abs(n)).sum((0, 1)) + 1e-40


def append(x, bits):
    """Scales [T][H] (float32) and unpacked codes [T][H][D] of rows x [T][H][D] (float32 values): each head on its own, NaNs ignored, a
    subnormal scale stored as zeros under 1, an infinite maximum as zeros under NaN."""
    x = np.asarray(x, np.float32)
    T, H, D = x.shape
    scales, codes = np.ones((T, H), np.float32), np.zeros((T, H, D), np.uint8)
    for t in range(T):
        for h in range(H):
            row = x[t, h]
            mx = np.float32(np.max(np.abs(row[~np.isnan(row)]), initial=0.0))
            if np.isinf(mx):
                scales[t, h] = np.nan
                continue
            s = np.float32(mx * np.float32(2.0 ** -(bits - 2)))
            if mx == 0 or s < np.finfo(np.float32).tiny:
                continue
            scales[t, h] = s
            codes[t, h] = R.quantize(row, s, bits, True)
    return scales, codes


def pack(codes, bits):
    return codes if bits == 8 else (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(codes, bits):
    return codes if bits == 8 else np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])


def read(codes, scales, bits, table, tokens, head):
    """Values [tokens][D] of one head from the pages of a table."""
    pages = np.asarray(table[: -(-tokens // codes.shape[2])], np.int64)
    c = unpack(codes[pages, head].reshape(-1, codes.shape[-1])[:tokens], bits)
    return R.codebook(bits, True).astype(np.float64)[c] * scales[pages, head].reshape(-1)[:tokens, None].astype(np.float64)


def attention(q, cache, tables, lengths, starts, causal, scale, dtype, prefix=None):
    """(out, bound).  q [T][Hq][D] float64; cache = (k_codes, k_scales, v_codes, v_scales, k_bits, v_bits) arrays; prefix = (tables,
    lengths, starts) or None.

    Bound.  A score is a sum of D exact products in fp32 and is scaled twice: (D + 8) roundings of the sum of their sizes; queries in
    fp32 are taken as 22 bits first.  A probability is exp2 of a difference: the error of the scores twice, 2 roundings of
    the exponential (its argument, times |score| at most, is one more), and 2^-11 (fp32 results: 2^-20) where it becomes an
    operand.  The sums over the keys lose a rounding a key at most.  Then the type's own rounding."""
    k, ks, v, vs, kb, vb = cache
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, bound = np.zeros((T, Hq, D)), np.full((T, Hq, D), TINY[dtype])
    operand = 2.0 ** -20 if dtype == "fp32" else 2.0 ** -11
    group_of = {}
    if prefix is not None:
        for g in range(len(prefix[1])):
            for s in range(prefix[2][g], prefix[2][g + 1]):
                group_of[s] = g
    for s in range(len(lengths)):
        a, b = (s, s + 1) if starts is None else (starts[s], starts[s + 1])
        n, L, g = b - a, int(lengths[s]), group_of.get(s)
        P = 0 if g is None else int(prefix[1][g])
        for head in range(Hkv):
            keys, values = (read(c, sc, bits, tables[s], L, head) for c, sc, bits in ((k, ks, kb), (v, vs, vb)))
            if P:
                keys = np.concatenate((read(k, ks, kb, prefix[0][g], P, head), keys))
                values = np.concatenate((read(v, vs, vb, prefix[0][g], P, head), values))
            for i in range(n):
                seen = P + (max(0, L - (n - 1 - i)) if causal else L)
                if not seen:
                    continue
                for h in range(head * G, head * G + G):
                    x = q[a + i, h]
                    score = keys[:seen] @ x * scale
                    size = np.abs(keys[:seen]) @ np.abs(x) * abs(scale)
                    off = ((D + 8) * U + (2.0 ** -22 if dtype == "fp32" else 0.0)) * size.max() + 2 * U * np.abs(score).max() + 4 * U
                    p = np.exp(score - score.max())
                    p /= p.sum()
                    out[a + i, h] = p @ values[:seen]
                    bound[a + i, h] += (p @ np.abs(values[:seen])) * (4 * off + operand + 2 * (seen + 16) * U) + HALF_ULP[dtype] * np.abs(out[a + i, h])
    return out, bound
