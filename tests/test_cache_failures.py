"""Calls of the pool's book-keeping that fail on their way: nothing has changed then (no GPU)."""
import copy

import pytest

from paper_2510_18121_amd.cache import KVCache, Sequences


def state(s):
    return copy.deepcopy((s.lengths, s.pages, s.uses, s.free_pages))


def forked(n_pages=12):
    s = Sequences(n_pages=n_pages)
    a, b = s.add(), s.add()
    s.extend([a, b], [130, 64])
    return s, a, b, s.fork(a)


def test_a_copy_that_fails_changes_nothing():
    s, a, b, c = forked()
    before, asked = state(s), []

    def fail(src, dst):
        asked.append((src, dst))
        raise RuntimeError("no launch")

    s._copy = fail
    for seqs, rows in (([c], [1]), ([b, a, c], [7, 100, 200])):
        with pytest.raises(RuntimeError):
            s.extend(seqs, rows)
        assert state(s) == before
    del s._copy  # (the method is there again: without caches it copies nothing)
    _, _, table = s.extend([c], [1])
    assert asked[0] == ([2], [4]) and table.tolist() == [[0, 1, 4]]


def test_arrays_that_fail_change_nothing():
    s, a, b, c = forked()
    before = state(s)
    with pytest.raises(RuntimeError):
        s.extend([c, b], [1, 300], device="no such device")
    assert state(s) == before
    start, lens, table = s.extend([c, b], [1, 300])
    assert start.tolist() == [0, 1, 301] and lens.tolist() == [131, 364] and table.tolist() == [[0, 1, 4, -1, -1, -1], [3, 5, 6, 7, 8, 9]]
    assert s.free_pages == [11, 10] and s.uses == [2, 2] + [1] * 8 + [0, 0]


def test_a_copy_that_fails_leaves_the_pool_as_it_was_before_a_compaction():
    s, a, b, c = forked()
    s.free(b)
    s.extend([a], [200])
    before = state(s)

    def fail(src, dst):
        raise RuntimeError("no launch")

    s._copy = fail
    with pytest.raises(RuntimeError):
        s.compact()
    assert state(s) == before


def test_a_pool_larger_than_a_cache_is_refused():
    """Tokens of pages that a cache does not have would be dropped without a word."""
    small, large = (KVCache.empty(n, 1, 64, "cpu") for n in (4, 6))
    assert len(Sequences([large, small]).free_pages) == 4 and len(Sequences([large, small], n_pages=3).free_pages) == 3
    for caches, n in (([small], 5), ([large, small], 6), ([], -1), ([small], -1)):
        with pytest.raises(ValueError):
            Sequences(caches, n_pages=n)
    with pytest.raises(TypeError):
        Sequences([small], n_pages=2.5)
