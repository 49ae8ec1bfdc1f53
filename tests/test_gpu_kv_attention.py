"""Attention over the cache of codes against 64 bits: widths, heads, types, lengths from nothing to several chunks, queries from one
to a chunk of a prompt, shared prefixes, places that hold NaN behind every end, refusals."""
import numpy as np
import pytest
import torch

from paper_2302_12510_amd import binding as B
from kv_util import World, check_attention, i32, typed

pytestmark = pytest.mark.gpu

LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 100, 127, 128, 129, 300, 511, 700]


@pytest.mark.parametrize("bits", [(8, 8), (8, 4), (4, 8), (4, 4)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_one_token_of_each_sequence(bits, D, dtype):
    rng = np.random.default_rng(D + bits[0] + 2 * bits[1])
    check_attention(rng, World(rng, LENGTHS, 2, D, bits, 16), None, 8, dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
def test_pages_of_any_size(page):
    rng = np.random.default_rng(page)
    check_attention(rng, World(rng, [page - 1, page, page + 1, 2 * page + 5, 3], 1, 64, (8, 4), page), None, 3, "fp16")


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 16, 17, 33])
def test_heads_that_share_a_key_head(group):
    rng = np.random.default_rng(group)
    check_attention(rng, World(rng, [5, 130, 257], 2, 64, (8, 8), 32), None, 2 * group, "bf16")


@pytest.mark.parametrize("bits", [(8, 8), (4, 4), (8, 4)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_several_tokens_of_each_sequence(bits, D, dtype, causal):
    rng = np.random.default_rng(D + bits[0])
    # more tokens than the cache holds: those in front see nothing
    new = [1, 2, 5, 0, 40, 17, 3]
    check_attention(rng, World(rng, [1, 200, 5, 9, 300, 17, 1], 2, D, bits, 16), new, 6, dtype, causal)


@pytest.mark.parametrize("n", [31, 64, 65, 127, 128, 129, 200])
@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
def test_chunks_of_a_prompt(n, dtype):
    rng = np.random.default_rng(n)
    check_attention(rng, World(rng, [n, n + 77, 2 * n + 1], 1, 128, (8, 8), 32), [n, n, n - 30], 3, dtype)


@pytest.mark.parametrize("D,dtype", [(64, "fp16"), (64, "fp32"), (128, "bf16"), (256, "fp16")])
@pytest.mark.parametrize("sequences,heads,n", [(32, 8, 20), (70, 4, 18), (5, 16, 150), (33, 9, 17)])
def test_more_tiles_of_rows_than_the_device_holds(D, dtype, sequences, heads, n):
    """Tiles are shared out whole but for the last ones, which are cut along the keys; which ones the numbers of queries say."""
    rng = np.random.default_rng(sequences + D)
    new = [int(x) for x in rng.integers(0, n + 1, sequences)]
    new[sequences // 2] = n
    lengths = [max(0, c + int(rng.integers(-3, 60))) if i % 5 else int(rng.integers(0, 300)) for i, c in enumerate(new)]
    check_attention(rng, World(rng, lengths, heads, D, (8, 4), 16), new, 2 * heads, dtype)


@pytest.mark.parametrize("D,bits,dtype", [(64, (4, 4), "fp16"), (128, (8, 8), "bf16"), (128, (4, 8), "fp32"), (256, (8, 4), "bf16")])
@pytest.mark.parametrize("new", [None, [1, 3, 0, 2, 30, 4, 1]])
def test_shared_prefix(D, bits, dtype, new):
    rng = np.random.default_rng(D)
    world = World(rng, [0, 3, 40, 200, 33, 64, 1], 2, D, bits, 16, prefixes=[700, 0, 33])
    check_attention(rng, world, new, 8, dtype, sizes=[4, 1, 2])


def test_many_sequences_share_a_prefix():
    rng = np.random.default_rng(5)
    world = World(rng, [int(x) for x in rng.integers(0, 40, 50)], 2, 128, (8, 8), 16, prefixes=[1000])
    check_attention(rng, world, None, 8, "bf16", sizes=[50])
    check_attention(rng, world, None, 8, "fp32", sizes=[50])


@pytest.mark.parametrize("D,dtype", [(64, "fp32"), (128, "bf16"), (256, "fp16"), (256, "fp32")])
@pytest.mark.parametrize("own,prefix", [([5, 0, 300], [128]), ([5, 0, 300], [2900]), ([700, 0, 520], [1300]), ([513, 1, 2], [0])])
@pytest.mark.parametrize("new", [None, [2, 5, 0], [40, 1, 0]])
def test_prefixes_of_few_and_of_many_parts(D, dtype, own, prefix, new):
    """Own tokens that are joined with the prefix in place, and those that a pass of its own joins; queries in front of the own tokens."""
    rng = np.random.default_rng(len(own) + own[0] + prefix[0] + D)
    check_attention(rng, World(rng, own, 2, D, (4, 8), 32, prefixes=prefix), new, 6, dtype, sizes=[3])


def test_prefix_of_a_group_with_more_queries_than_said():
    """Queries past max_queries get no prefix, and the flag says so; the others are as they were."""
    rng = np.random.default_rng(13)
    world = World(rng, [20, 30, 40], 1, 64, (8, 8), 16, prefixes=[100])
    q, _ = typed(rng.standard_normal((3, 2, 64)), "fp32")
    args = (q, world.cache(), i32(world.tables), i32(world.lengths))
    prefix = lambda n: B.SharedPrefix(i32(world.prefix_tables), i32(world.prefix_lengths), i32([0, 3]), n)  # noqa: E731
    want, alone = B.dybit_kv_attention(*args, prefix=prefix(3)), B.dybit_kv_attention(*args)
    assert B.dybit_get_last_async_error() == B.OK
    got = B.dybit_kv_attention(*args, prefix=prefix(2))
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG
    assert torch.equal(got[:2], want[:2])
    torch.testing.assert_close(got[2], alone[2], rtol=1e-5, atol=1e-6)


def test_groups_that_leave_sequences_out():
    rng = np.random.default_rng(6)
    world = World(rng, [10, 20, 30, 40], 1, 64, (8, 8), 16, prefixes=[100])
    q, q64 = typed(rng.standard_normal((4, 2, 64)), "fp32")
    from oracle import kv_ref as K
    from kv_util import within
    prefix = (world.prefix_tables, world.prefix_lengths, np.array([1, 3]))
    out = B.dybit_kv_attention(q, world.cache(), i32(world.tables), i32(world.lengths),
                               prefix=B.SharedPrefix(i32(prefix[0]), i32(prefix[1]), i32(prefix[2]), 2))
    want, bound = K.attention(q64, world.arrays, world.tables, world.lengths, None, True, 64 ** -0.5, "fp32", prefix)
    within(out, want, bound)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_long_sequence_in_many_parts(dtype):
    rng = np.random.default_rng(7)
    for lengths, max_length in (([9000, 1], 0), ([9000, 4097], 9100), ([20000], 0)):
        check_attention(rng, World(rng, lengths, 1, 64, (8, 4), 128), None, 4, dtype, max_length=max_length)


@pytest.mark.parametrize("strided", [1, 2, 9])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_strided_queries(strided, dtype):
    rng = np.random.default_rng(strided)
    check_attention(rng, World(rng, [40, 100], 2, 64, (8, 8), 16), [2, 30], 4, dtype, strided=strided)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_queries_and_scales_of_extreme_size(dtype):
    """Rows of queries from the smallest normals up, value scales over forty powers of two, one token far above the others."""
    rng = np.random.default_rng(8)
    world = World(rng, [300, 64], 1, 64, (8, 8), 16, spread=False)
    live = ~np.isnan(world.vs)
    world.vs[live] *= 2.0 ** rng.integers(-20, 21, live.sum())
    check_attention(rng, world, None, 2, dtype, scale=30.0)
    q, q64 = typed(np.stack([rng.standard_normal((2, 64)) * (1e-30 if dtype != "fp16" else 1e-7), np.zeros((2, 64))]), dtype)
    from oracle import kv_ref as K
    from kv_util import within
    out = B.dybit_kv_attention(q, world.cache(), i32(world.tables), i32(world.lengths), scale=1.0)
    want, bound = K.attention(q64, world.arrays, world.tables, world.lengths, None, True, 1.0, dtype)
    within(out, want, bound)


def test_peaked_scores():
    """One key that takes the whole row, met first, last and in the middle; scores of thousands."""
    rng = np.random.default_rng(9)
    for at in (0, 150, 299):
        world = World(rng, [300], 1, 64, (8, 8), 16, spread=False)
        world.ks[world.tables[0][at // 16], 0, at % 16] = 50.0
        check_attention(rng, world, None, 2, "fp32", scale=1.0)


def test_not_a_number_that_is_seen_stays_one():
    rng = np.random.default_rng(10)
    world = World(rng, [64, 64, 64], 1, 64, (8, 8), 16)
    q, _ = typed(rng.standard_normal((3, 2, 64)), "fp32")
    cache = world.cache()
    cache.k_scales[int(world.tables[0][1]), 0, 3] = float("nan")
    cache.v_scales[int(world.tables[1][2]), 0, 5] = float("nan")
    q[2, 1, 7] = float("nan")
    out = B.dybit_kv_attention(q, cache, i32(world.tables), i32(world.lengths))
    assert out[0].isnan().all() and out[1].isnan().all() and out[2, 1].isnan().all() and not out[2, 0].isnan().any()


def test_pages_and_lengths_out_of_range_are_left_out():
    rng = np.random.default_rng(11)
    world = World(rng, [64, 64], 1, 64, (8, 8), 16)
    q, _ = typed(rng.standard_normal((2, 2, 64)), "fp32")
    cache, tables = world.cache(), world.tables.copy()
    assert B.dybit_get_last_async_error() == B.OK
    good = B.dybit_kv_attention(q, cache, i32(tables), i32([64, 48]))
    tables[1, 3] = 1 << 20
    out = B.dybit_kv_attention(q, cache, i32(tables), i32([64, 64]))
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG
    assert torch.equal(out[0], good[0])
    torch.testing.assert_close(out[1], good[1], rtol=1e-5, atol=1e-6)
    out = B.dybit_kv_attention(q, cache, i32(world.tables), i32([1 << 30, -5]))
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG
    torch.testing.assert_close(out[0], good[0], rtol=1e-5, atol=1e-6)
    assert (out[1] == 0).all()
    B.dybit_kv_attention(q, cache, i32(world.tables), i32([4, 4]), i32([0, 7, -3]), max_queries=2)
    assert B.dybit_get_last_async_error() == B.ERR_INVALID_ARG


def test_nothing_to_do_and_an_empty_pool():
    cache = B.KVCache(*(torch.empty(0, 2, 16, w, dtype=d, device="cuda").squeeze(-1) if w == 1 else torch.empty(0, 2, 16, w, dtype=d, device="cuda")
                        for w, d in ((64, torch.uint8), (1, torch.float32), (32, torch.uint8), (1, torch.float32))), 8, 4)
    q = torch.randn(3, 4, 64, device="cuda")
    out = B.dybit_kv_attention(q, cache, i32(np.zeros((3, 0))), i32([0, 0, 0]))
    assert (out == 0).all() and B.dybit_get_last_async_error() == B.OK
    assert B.dybit_kv_attention(q[:0], cache, i32(np.zeros((0, 0))), i32([])).shape == (0, 4, 64)


def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(12)
    world = World(rng, [700, 300, 2], 2, 128, (8, 8), 64, prefixes=[500])
    q, _ = typed(rng.standard_normal((3, 8, 128)), "bf16")
    cache, tables, lengths = world.cache(), i32(world.tables), i32(world.lengths)
    prefix = B.SharedPrefix(i32(world.prefix_tables), i32(world.prefix_lengths), i32([0, 3]), 3)
    want = B.dybit_kv_attention(q, cache, tables, lengths, prefix=prefix)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.dybit_kv_attention(q, cache, tables, lengths, prefix=prefix, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        B.dybit_kv_attention(q, cache, tables, lengths, prefix=prefix, out=out)
    for i in range(3):
        q.copy_(torch.randn_like(q))
        lengths.copy_(i32([700 - 100 * i, 300, 2 - i]))
        want = B.dybit_kv_attention(q, cache, tables, lengths, prefix=prefix)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
@pytest.mark.parametrize("n", [1, 9, 40])
def test_wide_heads_over_long_and_short_sequences(dtype, n):
    """Few and many rows of 256 dims: workgroups that hold a compute unit alone, chunks in several rounds."""
    rng = np.random.default_rng(n)
    check_attention(rng, World(rng, [9000, 70, 1, 4100], 1, 256, (8, 4), 64), [n, min(n, 30), 1, n], 3, dtype)


@pytest.mark.parametrize("D,dtype", [(128, "fp32"), (256, "fp32"), (128, "bf16")])
def test_many_short_sequences_beside_a_long_one(D, dtype):
    """Nearly as many tiles as the device holds, of which one is long: it is cut into parts all the same."""
    rng = np.random.default_rng(D)
    lengths = [5200] + [int(x) for x in rng.integers(1, 60, 29)]
    check_attention(rng, World(rng, lengths, 7, D, (4, 8), 32), [34] + [int(x) for x in rng.integers(0, 20, 29)], 14, dtype)
