"""Helpers for the tests of the key/value cache (not collected by pytest)."""
import numpy as np
import torch

from oracle import kv_ref as K
from paper_2302_12510_amd import binding as B

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def typed(x, dtype):
    """(device tensor of the type, its values as float64)."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DTYPES[dtype])
    return t.cuda(), t.double().numpy()


def inside_larger(t, extra_heads=3, pad=0):
    """The same tensor as a view of a larger one: other strides by token and by head, other heads around it."""
    T, H, D = t.shape
    big = torch.full((T, H + extra_heads, D + pad), float("nan"), dtype=t.dtype, device=t.device)
    view = big[:, 1:1 + H, :D]
    view.copy_(t)
    return view


def within(got, want, bound, what=""):
    got = got.double().cpu().numpy()
    err = np.abs(got - want)
    bad = ~(err <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(np.isnan(err), np.inf, err - bound)), err.shape)
        raise AssertionError(f"{what} {bad.sum()} of {bad.size} outside; worst at {i}: got {got[i]!r} want {want[i]!r} bound {bound[i]:.3e}")


class World:
    """A pool of pages filled for some sequences (and prefixes), everything else in it poisoned: scales NaN, codes random."""

    def __init__(self, rng, lengths, heads, D, bits, page, prefixes=(), spread=True):
        counts = [-(-n // page) for n in list(lengths) + list(prefixes)]
        pages = sum(counts) + 3
        order = rng.permutation(pages)
        kb, vb = bits
        self.k = rng.integers(0, 256, (pages, heads, page, D * kb // 8), dtype=np.uint8)
        self.v = rng.integers(0, 256, (pages, heads, page, D * vb // 8), dtype=np.uint8)
        self.ks = np.full((pages, heads, page), np.nan, np.float32)
        self.vs = np.full((pages, heads, page), np.nan, np.float32)
        tables, at = [], 0
        width = max(1, max(counts))
        for n, c in zip(list(lengths) + list(prefixes), counts):
            row = np.full(width, -1, np.int32)
            row[:c] = order[at:at + c]
            at += c
            for t in range(n):
                p, i = row[t // page], t % page
                self.ks[p, :, i] = 0.02 * rng.uniform(0.5, 2, heads) * (2.0 ** rng.integers(-3, 4) if spread else 1)
                self.vs[p, :, i] = 0.03 * rng.uniform(0.5, 2, heads) * (2.0 ** rng.integers(-6, 7) if spread else 1)
            tables.append(row)
        n = len(lengths)
        self.lengths = np.array(lengths, np.int32)
        self.tables = np.array(tables[:n], np.int32).reshape(n, width)
        self.prefix_lengths = np.array(prefixes, np.int32)
        self.prefix_tables = np.array(tables[n:], np.int32).reshape(len(prefixes), width)
        self.arrays = (self.k, self.ks, self.v, self.vs, kb, vb)

    def cache(self):
        return B.KVCache(*(torch.from_numpy(a).cuda() for a in self.arrays[:4]), *self.arrays[4:])


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def check_attention(rng, world, new, Hq, dtype, causal=True, sizes=None, max_length=0, scale=None, strided=False):
    """One call against the oracle; `new`: query tokens of each sequence, None for one each without starts."""
    D, Hkv = world.k.shape[-1] * 8 // world.arrays[4], world.k.shape[1]
    n = len(world.lengths)
    starts = None if new is None else np.concatenate(([0], np.cumsum(new)))
    T = n if new is None else int(starts[-1])
    q, q64 = typed(rng.standard_normal((T, Hq, D)) * 2.0 ** rng.integers(-2, 2, (T, Hq, 1)), dtype)
    if strided:
        q = inside_larger(q, pad=strided - 1)
    scale = D ** -0.5 if scale is None else scale
    prefix = shared = None
    if sizes is not None:
        cuts = np.concatenate(([0], np.cumsum(sizes)))
        most = max(int(starts[b] - starts[a]) if new is not None else b - a for a, b in zip(cuts, cuts[1:]))
        prefix = (world.prefix_tables, world.prefix_lengths, cuts)
        shared = B.SharedPrefix(i32(world.prefix_tables), i32(world.prefix_lengths), i32(cuts), int(most))
    out = B.dybit_kv_attention(q, world.cache(), i32(world.tables), i32(world.lengths), None if new is None else i32(starts),
                               max_queries=1 if new is None else max(1, max(new)), max_length=max_length, causal=causal, scale=scale,
                               prefix=shared)
    assert out.dtype == q.dtype and out.shape == q.shape
    want, bound = K.attention(q64, world.arrays, world.tables, world.lengths, starts, causal, scale, dtype, prefix)
    assert B.dybit_get_last_async_error() == B.OK
    within(out, want, bound, f"{world.lengths} {new} {Hq} {dtype}")
    return out
