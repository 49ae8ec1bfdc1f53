"""Bookkeeping of the cache's pages, with the copies done on an array: what a sequence reads is always what was written to it."""
import numpy as np
import pytest

from paper_2302_12510_amd.kv_cache import PagePool, PoolFull


class Shadow:
    """A pool over an array of tokens, and what every sequence should hold."""

    def __init__(self, pages, page_tokens):
        self.pool, self.data, self.want = PagePool(pages, page_tokens), np.zeros((pages, page_tokens), np.int64), {}
        self.next = 1

    def copy(self, pairs):
        src, dst = [a for a, _ in pairs], [b for _, b in pairs]
        assert len(set(dst)) == len(dst) and not set(src) & set(dst)
        self.data[dst] = self.data[src]

    def extend(self, seq, n):
        slots = self.pool.extend(seq, n)
        assert slots.dtype == np.int64 and len(slots) == n
        values = np.arange(self.next, self.next + n)
        self.next += n
        self.data.reshape(-1)[slots] = values
        self.want[seq] = self.want.get(seq, []) + values.tolist()

    def check(self):
        seqs = list(self.want)
        table, tokens = self.pool.tables(seqs)
        for row, n, s in zip(table, tokens, seqs):
            used = -(-int(n) // self.pool.page_tokens)
            assert (row[used:] == -1).all() and (row[:used] >= 0).all()
            assert self.data[row[:used]].reshape(-1)[:n].tolist() == self.want[s]
        count = np.zeros(len(self.pool.owners), int)
        for s in seqs:
            for p in self.pool.pages(s):
                count[p] += 1
        assert (count == self.pool.owners).all() and self.pool.free_pages == (count == 0).sum()


@pytest.mark.parametrize("page", [1, 4, 16])
def test_random_use(page):
    rng = np.random.default_rng(page)
    w = Shadow(120, page)
    names = iter(range(10 ** 6))
    for _ in range(600):
        seqs = list(w.want)
        do = rng.choice(["add", "extend", "extend", "fork", "free", "compact"])
        try:
            if do == "add":
                s = next(names)
                w.pool.add(s)
                w.want[s] = []
            elif do == "extend" and seqs:
                w.extend(seqs[rng.integers(len(seqs))], int(rng.integers(0, 3 * page + 2)))
            elif do == "fork" and seqs:
                parent = seqs[rng.integers(len(seqs))]
                children = [next(names) for _ in range(rng.integers(0, 4))]
                w.copy(w.pool.fork(parent, children))
                for c in children:
                    w.want[c] = list(w.want[parent])
            elif do == "free" and seqs:
                s = seqs[rng.integers(len(seqs))]
                w.pool.free(s)
                del w.want[s]
            elif do == "compact":
                w.copy(w.pool.compact())
                used = (w.pool.owners > 0).sum()
                assert (w.pool.owners[:used] > 0).all()
        except PoolFull:
            pass
        w.check()


def test_full_pool_changes_nothing():
    w = Shadow(3, 4)
    w.pool.add("a")
    w.extend("a", 9)
    with pytest.raises(PoolFull):
        w.pool.extend("a", 5)
    with pytest.raises(PoolFull):
        w.pool.fork("a", ["b"])
    assert "b" not in w.pool
    w.check()
    w.extend("a", 3)
    w.copy(w.pool.fork("a", ["b"]))                               # whole pages only: shared, none taken
    w.want["b"] = list(w.want["a"])
    w.check()
    assert w.pool.pages("a") == w.pool.pages("b") and w.pool.free_pages == 0


def test_refusals():
    pool = PagePool(4, 4)
    pool.add(1)
    with pytest.raises(KeyError):
        pool.add(1)
    with pytest.raises(KeyError):
        pool.fork(1, [2, 2])
    with pytest.raises(KeyError):
        pool.fork(1, [1])
    with pytest.raises(KeyError):
        pool.extend(9)
    with pytest.raises(ValueError):
        pool.extend(1, -1)
    with pytest.raises(KeyError):
        pool.free(9)
    pool.extend(1, 9)
    with pytest.raises(ValueError):
        pool.tables([1], width=2)
    with pytest.raises(ValueError):
        PagePool(4, 0)
    assert pool.tables([])[0].shape == (0, 1)
