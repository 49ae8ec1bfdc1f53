"""Appending to the cache (bit exact) and copying its pages."""
import numpy as np
import pytest
import torch

from oracle import kv_ref as K
from paper_2302_12510_amd import binding as B
from kv_util import DTYPES, inside_larger

pytestmark = pytest.mark.gpu


def empty(pages, heads, page, D, kb, vb, layers=None):
    lead = (pages,) if layers is None else (layers, pages)
    return B.KVCache(torch.randint(0, 256, (*lead, heads, page, D * kb // 8), dtype=torch.uint8, device="cuda"),
                     torch.randn(*lead, heads, page, device="cuda"),
                     torch.randint(0, 256, (*lead, heads, page, D * vb // 8), dtype=torch.uint8, device="cuda"),
                     torch.randn(*lead, heads, page, device="cuda"), kb, vb)


def check_append(k, v, slots, cache):
    """The whole cache after the call: what was named holds the oracle's codes and scales, everything else what it held."""
    before = [t.cpu().numpy().copy() for t in cache[:4]]
    B.dybit_kv_append(k, v, torch.tensor(slots, dtype=torch.int64, device="cuda"), cache)
    page = cache.k_codes.shape[2]
    for x, codes, scales, bits in ((k, 0, 1, cache.k_bits), (v, 2, 3, cache.v_bits)):
        s, c = K.append(x.float().cpu().numpy(), bits)
        c = K.pack(c, bits)
        for t, slot in enumerate(slots):
            if 0 <= slot < cache.k_codes.shape[0] * page:
                before[codes][slot // page, :, slot % page] = c[t]
                before[scales][slot // page, :, slot % page] = s[t]
    for name, got, want in zip(cache._fields, cache[:4], before):
        np.testing.assert_array_equal(got.cpu().numpy(), want, err_msg=name)


@pytest.mark.parametrize("bits", [(8, 8), (8, 4), (4, 8), (4, 4)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_append(bits, D, dtype):
    rng = np.random.default_rng(D + bits[0])
    cache = empty(5, 3, 16, D, *bits)
    x = [torch.from_numpy(rng.standard_normal((21, 3, D)) * 2.0 ** rng.integers(-6, 7, (21, 3, 1))).to(DTYPES[dtype]).cuda() for _ in range(2)]
    check_append(*x, rng.permutation(80)[:21].tolist(), cache)
    assert B.dybit_get_last_async_error() == B.OK


@pytest.mark.parametrize("T", [0, 1, 2, 1000])
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_append_tokens_and_pages(T, page):
    rng = np.random.default_rng(T)
    cache = empty(1 + 1100 // page, 2, page, 64, 8, 4)
    x = [torch.from_numpy(rng.standard_normal((T, 2, 64))).float().cuda() for _ in range(2)]
    check_append(*x, rng.permutation(cache.k_codes.shape[0] * page)[:T].tolist(), cache)


@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_append_strided(pad, dtype):
    cache = empty(3, 2, 16, 64, 8, 4)
    x = [inside_larger(torch.randn(9, 2, 64, device="cuda").to(DTYPES[dtype]), pad=pad) for _ in range(2)]
    check_append(*x, list(range(20, 29)), cache)


@pytest.mark.parametrize("bits", [4, 8])
def test_append_ties_and_every_size(bits):
    """Values on the decision points of the codes, rows from subnormal to the largest floats, zeros, NaN."""
    from oracle import dybit_ref as R
    mid = R.midpoints(bits - 1)
    top = 2.0 ** (bits - 2)
    rows = []
    for scale in (1.0, 3.0, 2.0 ** -60, 2.0 ** 60, 2.0 ** -119, 2.0 ** 120, 1.1754944e-38, 1.5e-38, 2.0 ** 121):
        s = np.float64(np.float32(scale))
        for m in np.array_split(np.concatenate((mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9))), max(1, 3 * len(mid) // 60)):
            row = np.zeros(64)
            row[:len(m)] = m * s * np.where(np.arange(len(m)) % 2, -1, 1)
            row[63] = top * s
            rows.append(row)
    rows.append(np.zeros(64))
    rows.append(np.full(64, 1e-42))
    rows.append(np.full(64, 2e-37))
    rows.append(np.where(np.arange(64) % 3 == 0, np.nan, np.arange(64)))
    rows.append(np.full(64, np.nan))
    rows.append(np.full(64, -0.0))
    with np.errstate(over="ignore", under="ignore"):
        x = torch.from_numpy(np.array(rows).astype(np.float32)).cuda().view(-1, 1, 64).contiguous()
    x = x[torch.isfinite(x).logical_or(x.isnan()).all(-1).squeeze(1)]
    cache = empty(1 + len(x) // 64, 1, 64, 64, bits, 12 - bits)
    check_append(x, x.flip(0).contiguous(), list(range(len(x))), cache)
    assert B.dybit_get_last_async_error() == B.OK


def test_append_flags_what_cannot_be_stored():
    cache = empty(2, 1, 16, 64, 8, 8)
    x = torch.randn(4, 1, 64, device="cuda")
    y = x.clone()
    y[1, 0, 5] = float("-inf")
    check_append(x, y, [3, 4, 5, 6], cache)
    assert B.dybit_get_last_async_error() == B.ERR_BAD_SCALE
    check_append(x, x, [-1, 8, -(1 << 40), 9], cache)                            # skipped, no error
    assert B.dybit_get_last_async_error() == B.OK
    check_append(x, x, [32, 10, 1 << 40, 11], cache)                             # past the pool
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG


@pytest.mark.parametrize("layers", [None, 1, 3])
@pytest.mark.parametrize("heads,page,D,bits", [(1, 16, 64, (4, 4)), (3, 16, 64, (8, 4)), (8, 64, 128, (8, 8)), (2, 128, 256, (4, 8))])
@pytest.mark.parametrize("n", [0, 1, 7, 50])
def test_copy_pages(layers, heads, page, D, bits, n):
    rng = np.random.default_rng(n)
    cache = empty(101, heads, page, D, *bits, layers=layers)
    moved = rng.permutation(101)[:2 * n]
    want = [t.clone() for t in cache[:4]]
    at = (slice(None),) if layers else ()
    for w in want:
        w[(*at, torch.from_numpy(moved[n:]).cuda())] = w[(*at, torch.from_numpy(moved[:n]).cuda())]
    B.dybit_kv_copy_pages(cache, *(torch.tensor(m, dtype=torch.int32, device="cuda") for m in (moved[:n], moved[n:])))
    for got, w in zip(cache[:4], want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))
    assert B.dybit_get_last_async_error() == B.OK


def test_copy_pages_outside_the_pool():
    cache = empty(5, 1, 16, 64, 8, 8)
    want = [t.clone() for t in cache[:4]]
    for w in want:
        w[3] = w[1]
    B.dybit_kv_copy_pages(cache, *(torch.tensor(m, dtype=torch.int32, device="cuda") for m in ([1, 0, -1, 5], [3, 5, 4, 2])))
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG
    for got, w in zip(cache[:4], want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))


def test_refusals():
    cache = empty(4, 2, 16, 64, 8, 4)
    x = torch.randn(3, 2, 64, device="cuda")
    slots = torch.arange(3, device="cuda")
    table, one = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")

    def refused(status, call, *args, **kw):
        with pytest.raises(B.DybitError) as e:
            call(*args, **kw)
        assert e.value.status == status

    refused(B.ERR_INVALID_ARG, B.dybit_kv_append, x[:, :1], x[:, :1], slots, cache)            # other heads
    refused(B.ERR_INVALID_ARG, B.dybit_kv_append, x, x.half(), slots, cache)                   # two types
    refused(B.ERR_INVALID_ARG, B.dybit_kv_append, x, x[:2], slots, cache)
    refused(B.ERR_UNSUPPORTED_BITS, B.dybit_kv_append, x, x, slots, empty(4, 2, 16, 64, 6, 4))
    refused(B.ERR_INVALID_ARG, B.dybit_kv_append, x, x, slots, empty(4, 2, 24, 64, 8, 4))      # a page of 24 tokens
    refused(B.ERR_INVALID_ARG, B.dybit_kv_append, x[..., :32], x[..., :32], slots, empty(4, 2, 16, 32, 8, 8))
    refused(B.ERR_INVALID_ARG, B.dybit_kv_append, x, x, slots, empty(4, 2, 16, 64, 8, 4, layers=2))
    refused(B.ERR_INVALID_ARG, B.dybit_kv_attention, x[:, :1].contiguous(), cache, table, one)  # fewer query heads than key heads
    refused(B.ERR_INVALID_ARG, B.dybit_kv_attention, torch.randn(3, 3, 64, device="cuda"), cache, table, one)
    refused(B.ERR_INVALID_ARG, B.dybit_kv_attention, x, cache, table, one, scale=float("inf"))
    refused(B.ERR_INVALID_ARG, B.dybit_kv_attention, x, cache, table, one, out=torch.empty(3, 2, 64, device="cuda", dtype=torch.half))
    refused(B.ERR_INVALID_ARG, B.dybit_kv_attention, x, cache, table, one, max_queries=-1)
    refused(B.ERR_INVALID_ARG, B.dybit_kv_copy_pages, cache, torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        B.dybit_kv_append(x, x, slots.int(), cache)
    with pytest.raises(TypeError):
        B.dybit_kv_append(x.double(), x.double(), slots, cache)
    with pytest.raises(TypeError):
        B.dybit_kv_attention(x, cache, table.long(), one)
    with pytest.raises(TypeError):
        B.dybit_kv_append(x, x, slots, cache._replace(k_scales=cache.k_scales.half()))
    with pytest.raises(ValueError):
        B.dybit_kv_append(x, x, slots[:2], cache)
    with pytest.raises(ValueError):
        B.dybit_kv_append(x, x, slots, cache._replace(v_scales=cache.v_scales[:2]))
    with pytest.raises(ValueError):
        B.dybit_kv_append(x.cpu(), x, slots, cache)
    with pytest.raises(ValueError):
        B.dybit_kv_append(x.transpose(1, 2), x, slots, cache)
    with pytest.raises(ValueError):
        B.dybit_kv_attention(x, cache, table[:2], one)
    with pytest.raises(ValueError):
        B.dybit_kv_attention(x, cache, table, one, torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        B.dybit_kv_attention(x, cache, table, one, prefix=B.SharedPrefix(table, one[:2], one, 3))
