"""The page bookkeeping (host only) against a plain model: who owns what, which copies a write needs, compaction."""
import ctypes
import random

import pytest

from paper_2608_15018_b200 import binding


class Model:
    """Every sequence as the content it should see: one token per position, pages as lists of tokens."""

    def __init__(self, n_pages, size):
        self.size, self.store = size, [[None] * size for _ in range(n_pages)]

    def copy(self, pairs):
        old = [list(p) for p in self.store]
        assert not {a for a, _ in pairs} & {b for _, b in pairs} and len({b for _, b in pairs}) == len(pairs)
        for a, b in pairs:
            self.store[b] = old[a]

    def write(self, pages, start, tokens):
        for i, t in enumerate(tokens):
            self.store[pages[(start + i) // self.size]][(start + i) % self.size] = t

    def read(self, pages, n):
        return [self.store[pages[i // self.size]][i % self.size] for i in range(n)]


@pytest.mark.parametrize("seed", range(12))
def test_random_histories_keep_every_sequence_apart(seed):
    rng = random.Random(seed)
    n_pages, size = rng.choice([8, 30, 100]), rng.choice([1, 4, 16])
    pool, model = binding.PagePool(n_pages, size), Model(n_pages, size)
    content, fresh = {}, iter(range(10 ** 9))
    for _ in range(400):
        act = rng.choice(["open", "fork", "write", "write", "write", "cut", "free", "compact", "rewrite"])
        if act == "open" and len(content) < 12:
            s = pool.open()
            assert s not in content
            content[s] = []
        elif not content:
            continue
        s = rng.choice(list(content)) if content else None
        if act == "fork" and len(content) < 12:
            t = pool.fork(s)
            assert t not in content
            content[t] = list(content[s])
        elif act in ("write", "rewrite"):
            start = len(content[s]) if act == "write" else rng.randint(0, len(content[s]))
            tokens = [next(fresh) for _ in range(rng.randint(0, 3 * size))]
            if act == "rewrite":                                  # in the middle, what lies behind stays
                tokens = tokens[:len(content[s]) - start]
            before = (pool.pages(s), pool.free_pages())
            try:
                pairs = pool.reserve(s, start, start + len(tokens))
            except binding.S2MoEError as e:
                assert e.status == binding.ENOMEM and before == (pool.pages(s), pool.free_pages())
                continue
            model.copy(pairs)
            model.write(pool.pages(s), start, tokens)
            content[s][start:start + len(tokens)] = tokens
        elif act == "cut":
            n = rng.randint(0, len(content[s]))
            pool.truncate(s, n)
            del content[s][n:]
            assert len(pool.pages(s)) == (n + size - 1) // size
        elif act == "free":
            pool.free(s)
            del content[s]
        elif act == "compact":
            model.copy(pool.compact())
            used = {p for t in content for p in pool.pages(t)}
            assert used == set(range(len(used)))
        held = {p for t in content for p in pool.pages(t)}
        assert pool.free_pages() == n_pages - len(held)
        for t, tokens in content.items():
            assert model.read(pool.pages(t), len(tokens)) == tokens, (act, t)
    pool.close()


def test_forks_share_until_they_write():
    pool = binding.PagePool(10, 16)
    a = pool.open()
    assert pool.reserve(a, 0, 40) == [] and pool.pages(a) == [0, 1, 2]
    b = pool.fork(a)
    assert pool.pages(b) == [0, 1, 2] and pool.free_pages() == 7
    assert pool.reserve(b, 40, 41) == [(2, 3)] and pool.pages(b) == [0, 1, 3]       # the half filled page is copied
    assert pool.reserve(a, 40, 41) == []                                          # and its first owner keeps it
    pool.free(a)
    assert pool.free_pages() == 7 and pool.pages(b) == [0, 1, 3]
    assert pool.compact() == [(3, 2)] and pool.pages(b) == [0, 1, 2]


def test_refusals_change_nothing():
    lib = binding.load_library()
    for args in ((0, 16), (4, 0), (-1, 16)):
        with pytest.raises(binding.S2MoEError):
            binding.PagePool(*args)
    pool = binding.PagePool(4, 16)
    a = pool.open()
    pool.reserve(a, 0, 33)
    for call in (lambda: pool.reserve(a, 0, 65), lambda: pool.reserve(a, 2 ** 62, 2 ** 63 - 1), lambda: pool.reserve(a, 5, 4),
                 lambda: pool.reserve(a, -1, 4), lambda: pool.reserve(7, 0, 1), lambda: pool.fork(-1), lambda: pool.truncate(9, 0),
                 lambda: pool.truncate(a, -1), lambda: pool.free(3), lambda: pool.pages(2)):
        with pytest.raises(binding.S2MoEError):
            call()
        assert pool.pages(a) == [0, 1, 2] and pool.free_pages() == 1
    b = pool.fork(a)
    with pytest.raises(binding.S2MoEError):
        pool.reserve(b, 0, 33)                                   # three shared pages, one free
    assert pool.pages(b) == [0, 1, 2]
    n, pairs = ctypes.c_int32(0), (ctypes.c_int32 * 2)()
    assert lib.s2moe_pages_reserve(pool._h, b, 40, 41, 0, None, ctypes.byref(n)) == binding.ERANGE and n.value == 1
    assert pool.pages(b) == [0, 1, 2]
    assert lib.s2moe_pages_reserve(pool._h, b, 40, 41, 1, ctypes.cast(pairs, ctypes.c_void_p), ctypes.byref(n)) == binding.OK
    assert list(pairs) == [2, 3]
    assert lib.s2moe_pages_compact(pool._h, 0, None, ctypes.byref(n)) == binding.OK and n.value == 0
    pool.free(b)
    with pytest.raises(binding.S2MoEError):
        pool.free(b)
    assert lib.s2moe_pages_destroy(None) == binding.OK
    assert lib.s2moe_pages_open(None, ctypes.byref(n)) == binding.EINVAL
