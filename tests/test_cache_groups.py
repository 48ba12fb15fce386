"""Groups of sequences that share their first pages, and what attention over them refuses (no GPU)."""
import ctypes
import itertools

import numpy as np
import pytest

from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd.cache import CacheDesc, Sequences


def saved(common, cuts):
    """Pages not read again, of groups that begin at `cuts`."""
    total = 0
    for a, b in zip(cuts, cuts[1:]):
        total += (b - a - 1) * min(common[a + 1:b], default=0)
    return total


@pytest.mark.parametrize("seed", range(30))
def test_groups_save_the_most(seed):
    rng = np.random.default_rng(seed)
    s, live = Sequences(n_pages=4000), []
    for _ in range(int(rng.integers(1, 8))):  # a forest of forks
        if not live or rng.random() < 0.3:
            live.append(s.add())
        else:
            live.append(s.fork(live[rng.integers(len(live))]))
        s.extend([live[-1]], [int(rng.integers(0, 700))])
    rows = [int(rng.integers(0, min(3, s.lengths[x]) + 1)) for x in live]
    start, pages = (x.tolist() for x in s.groups(live, rows))
    n = len(live)
    common = [0] * n
    for i in range(1, n):
        a, b = live[i - 1], live[i]
        top = min((s.lengths[a] - rows[i - 1]) // 64, (s.lengths[b] - rows[i]) // 64)
        while common[i] < top and s.pages[a][common[i]] == s.pages[b][common[i]]:
            common[i] += 1
    assert start[0] == 0 and start[-1] == n and len(pages) == len(start) - 1 and all(a < b for a, b in zip(start, start[1:]))
    for a, b, p in zip(start, start[1:], pages):
        assert p == (min(common[a + 1:b]) if b - a > 1 else 0)
        assert all(s.pages[live[i]][:p] == s.pages[live[a]][:p] and s.lengths[live[i]] - rows[i] >= 64 * p for i in range(a, b))
    most = max(saved(common, (0, *cut, n)) for k in range(n) for cut in itertools.combinations(range(1, n), k))
    assert saved(common, start) == most


def test_forks_of_a_prompt():
    s = Sequences(n_pages=100)
    a = s.add()
    s.extend([a], [200])
    forks = [s.fork(a) for _ in range(3)]
    s.extend(forks, [1, 2, 3])
    assert [x.tolist() for x in s.groups(forks, [1, 2, 3])] == [[0, 3], [3]]
    assert [x.tolist() for x in s.groups(forks + [a], [1, 2, 3, 1])] == [[0, 4], [3]]
    assert [x.tolist() for x in s.groups([a, forks[0]], [100, 1])] == [[0, 2], [1]]  # rows of a that sit inside: one page is seen by all
    b = s.add()
    s.extend([b], [64])
    assert [x.tolist() for x in s.groups([forks[0], b, forks[1]], [1, 1, 1])] == [[0, 1, 2, 3], [0, 0, 0]]
    assert [x.tolist() for x in s.groups([], [])] == [[0], []]
    with pytest.raises(ValueError):
        s.groups([a], [])


def test_pages_behind_a_window_are_not_shared():
    s = Sequences(n_pages=100)
    a = s.add()
    s.extend([a], [1000])
    s.leave_window(a, 200, sinks=70)
    assert [x.tolist() for x in s.groups([a, s.fork(a)], [1, 1])] == [[0, 2], [2]]


PTR = 1 << 20


def call(cache=None, batch=None, groups=None, hq=8, q=PTR, o=PTR, ws=PTR, ws_bytes=1 << 40):
    c, b, g = CacheDesc(4, 2, 128, PTR, PTR, PTR, PTR), B.CacheBatch(2, 3, 10, PTR, PTR, PTR), B.CacheGroups(1, PTR, PTR)
    for t, fields in ((c, cache), (b, batch), (g, groups)):
        for name, x in (fields or {}).items():
            setattr(t, name, x)
    return B.lib().ca_cache_attend_shared(ctypes.byref(c), ctypes.byref(b), ctypes.byref(g), hq, 0.0, q, o, None, ws, ws_bytes, None)


BAD, NOT, ROOM = B.CA_ERR_INVALID_ARG, B.CA_ERR_UNSUPPORTED, B.CA_ERR_WORKSPACE


@pytest.mark.parametrize("want,kw", [
    (NOT, {"cache": {"head_dim": 96}}), (BAD, {"cache": {"k_scale": None}}), (NOT, {"batch": {"n_seqs": 4097}}), (BAD, {"batch": {"q_start": None}}),
    (BAD, {"groups": {"n_groups": -1}}), (BAD, {"groups": {"n_groups": 3}}), (BAD, {"groups": {"group_start": None}}), (BAD, {"groups": {"prefix_pages": None}}),
    (NOT, {"hq": 7}), (NOT, {"hq": 0}), (BAD, {"q": None}), (BAD, {"o": PTR + 8}), (ROOM, {"ws": None}), (ROOM, {"ws_bytes": 1000}), (ROOM, {"ws": PTR + 16}),
    (NOT, {"batch": {"total_rows": 1 << 24, "table_width": 1 << 12}})])
def test_calls_that_are_refused(want, kw):
    assert call(**kw) == want
    assert B.lib().ca_last_error()


def test_null_groups_and_nothing_to_do():
    c, b = CacheDesc(4, 2, 128, PTR, PTR, PTR, PTR), B.CacheBatch(2, 3, 10, PTR, PTR, PTR)
    assert B.lib().ca_cache_attend_shared(ctypes.byref(c), ctypes.byref(b), None, 8, 0.0, PTR, PTR, None, PTR, 1 << 40, None) == BAD
    assert call(batch={"total_rows": 0}) == B.CA_OK
    assert call(batch={"n_seqs": 0}, groups={"n_groups": 0}) == B.CA_OK


def test_workspace_grows_with_the_rows():
    c = CacheDesc(4, 8, 128, PTR, PTR, PTR, PTR)
    sizes = []
    for rows in (0, 1, 64, 1000):
        n = ctypes.c_size_t()
        assert B.lib().ca_cache_attend_shared_workspace_bytes(ctypes.byref(c), 32, rows, ctypes.byref(n)) == B.CA_OK
        sizes.append(n.value)
    assert sizes[0] < sizes[1] <= sizes[2] < sizes[3] and sizes[3] - sizes[0] >= 2 * 1000 * 32 * (128 + 4) * 4
    assert B.lib().ca_cache_attend_shared_workspace_bytes(ctypes.byref(c), 33, 1, ctypes.byref(n)) == NOT
    assert B.lib().ca_cache_attend_shared_workspace_bytes(ctypes.byref(c), 32, -1, ctypes.byref(n)) == BAD
    assert B.lib().ca_cache_attend_shared_workspace_bytes(ctypes.byref(c), 32, 1, None) == BAD
