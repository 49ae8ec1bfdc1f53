"""The decoder that runs the cache's operators together, and the calls through both ways of marshalling."""
import pytest
import torch

from paper_2302_12510_amd import binding as B
from paper_2302_12510_amd.decoder import Config, Decoder, generate

pytestmark = pytest.mark.gpu


def close(a, b):
    """Results that differ by the order of sums: an 8-bit code of an input may then be its neighbour, 2^-6 of it; all of them in each of
    four products of two layers would be 8 * 2^-6 of the result."""
    assert (a - b).norm() <= 0.125 * b.norm()


def test_a_prompt_at_once_and_in_pieces_and_shared():
    config = Config(layers=2)
    tokens = torch.randint(0, config.vocabulary, (53,), generator=torch.Generator().manual_seed(3)).tolist()
    model = Decoder(config)
    store = model.store
    for s in ("whole", "pieces", "prefix", "tail"):
        store.add(s)
    want = model.step(["whole"], [tokens])
    for a, b in ((0, 20), (20, 21), (21, 40)):
        model.step(["pieces"], [tokens[a:b]])
    close(model.step(["pieces"], [tokens[40:]]), want)
    model.step(["prefix"], [tokens[:37]])
    close(model.step(["tail"], [tokens[37:]], "prefix"), want)
    store.fork("whole", ["left", "right"])
    assert torch.equal(*model.step(["left", "right"], [[5], [5]]))           # two rows of one call over two copies
    before = model.step(["left"], [[7]])
    store.free("pieces")
    store.free("prefix")
    assert store.compact()
    store.fork("right", ["again"])
    assert torch.equal(model.step(["right"], [[7]]), before) and torch.equal(model.step(["again"], [[7]]), before)
    assert B.dybit_get_last_async_error() == B.OK


def test_branches():
    model = Decoder(Config(layers=1, pages=64))
    answers = generate(model, list(range(33)), length=6)
    assert sorted(answers) == [("fork", 0), ("fork", 1), ("tail", 0), ("tail", 1)] and all(len(a) == 7 for a in answers.values())
    assert B.dybit_get_last_async_error() == B.OK


def test_both_ways_of_marshalling(monkeypatch):
    results = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(B, "_native_module", B._Ctypes())
        torch.manual_seed(0)
        qkv = torch.randn(40, 8, 64, device="cuda")
        w, angle = torch.rand(64, device="cuda"), torch.rand(50, 32, device="cuda")
        args = (qkv[:, :4], qkv[:, 4:6], w, w, torch.arange(40, device="cuda"), angle.cos(), angle.sin())
        q, k = B.dybit_head_norm_rope(*args)
        grads = B.dybit_head_norm_rope_bwd(q, k, *args)
        new = lambda *n, d: torch.zeros(2, 9, 2, 16, *n, dtype=d, device="cuda")  # noqa: E731
        cache = B.KVCache(new(64, d=torch.uint8), new(d=torch.float32), new(32, d=torch.uint8), new(d=torch.float32), 8, 4)
        B.dybit_kv_append(k, qkv[:, 6:], torch.arange(40, device="cuda"), cache.layer(1))
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        B.dybit_kv_copy_pages(cache, i32([0, 1]), i32([7, 8]))
        prefix = B.SharedPrefix(i32([[7, 8]]), i32([20]), i32([0, 2]), 5)
        out = B.dybit_kv_attention(q[:5], cache.layer(1), i32([[0], [2]]), i32([16, 8]), i32([0, 2, 5]), max_queries=3, prefix=prefix)
        results.append((q, k, *grads, *cache[:4], out))
    for a, b in zip(*results):
        assert torch.equal(a, b)
