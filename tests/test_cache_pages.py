"""The host's book-keeping of a cache's pages, and what the cache's calls refuse (no GPU)."""
import ctypes
import random

import pytest
import torch

from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd.cache import CacheDesc, KVCache, OutOfPages, Sequences


def consistent(s):
    uses = [0] * len(s.uses)
    for seq, pages in s.pages.items():
        held = [p for p in pages if p >= 0]
        assert len(set(held)) == len(held) and len(pages) == -(-s.lengths[seq] // 64)
        for p in held:
            uses[p] += 1
    assert uses == s.uses
    assert sorted(s.free_pages) == [p for p, u in enumerate(uses) if u == 0]


def test_pages_are_handed_out_shared_copied_and_given_back():
    s = Sequences(n_pages=8)
    a, b = s.add(), s.add()
    start, lens, table = s.extend([a, b], [130, 64])
    assert start.tolist() == [0, 130, 194] and lens.tolist() == [130, 64]
    assert table.tolist() == [[0, 1, 2], [3, -1, -1]]
    c = s.fork(a)
    assert s.pages[c] == [0, 1, 2] and s.uses[:4] == [2, 2, 2, 1]
    moved = []
    s._copy = lambda src, dst: moved.append((src, dst))
    s.extend([c], [1])  # the shared last page is copied, full ones stay shared
    assert moved == [([2], [4])] and s.pages[c] == [0, 1, 4] and s.uses[:5] == [2, 2, 1, 1, 1]
    s.extend([b], [1])
    assert moved[1:] == [([], [])] and s.pages[b] == [3, 5]
    consistent(s)
    s.free(a)
    assert s.uses[2] == 0 and s.uses[0] == 1
    consistent(s)


def test_both_forks_extended_at_once_copy_the_shared_page_once():
    s = Sequences(n_pages=8)
    a = s.add()
    s.extend([a], [10])
    c = s.fork(a)
    moved = []
    s._copy = lambda src, dst: moved.append((src, dst))
    s.extend([a, c], [1, 1])
    assert moved == [([0], [1])] and sorted((s.pages[a], s.pages[c])) == [[0], [1]]
    consistent(s)


def test_a_full_pool_refuses_and_changes_nothing():
    s = Sequences(n_pages=3)
    a = s.add()
    s.extend([a], [129])
    c = s.fork(a)
    before = (dict(s.lengths), {k: list(v) for k, v in s.pages.items()}, list(s.uses), list(s.free_pages))
    for seqs, rows in (([a], [64]), ([c], [1]), ([a, c], [1, 1])):
        with pytest.raises(OutOfPages):
            s.extend(seqs, rows)
        assert before == (s.lengths, s.pages, s.uses, s.free_pages)
    for seqs, rows in (([a, a], [1, 1]), ([a], [-1]), ([a], [1, 2])):
        with pytest.raises(ValueError):
            s.extend(seqs, rows)
    with pytest.raises(KeyError):
        s.extend([99], [1])
    with pytest.raises(TypeError):
        s.extend([a], [1.5])
    assert before == (s.lengths, s.pages, s.uses, s.free_pages)


@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 0), (65, 3), (200, 64), (130, 65)])
def test_pages_behind_the_window_are_let_go(window, sinks):
    for length in (1, 64, 65, 191, 192, 193, 500):
        s = Sequences(n_pages=10)
        a = s.add()
        s.extend([a], [length])
        s.leave_window(a, window, sinks)
        seen = {j // 64 for j in range(length) if length - j < window or j < sinks}  # by the next row, at position `length`
        assert {i for i, p in enumerate(s.pages[a]) if p >= 0} >= seen
        gone = [i for i, p in enumerate(s.pages[a]) if p < 0]
        assert all(i * 64 >= sinks and i * 64 + 63 <= length - window for i in gone)
        assert len(gone) >= max(0, (length - window + 1) // 64 - -(-sinks // 64))
        consistent_uses = [p for p in s.pages[a] if p >= 0]
        assert sorted(consistent_uses + s.free_pages) == list(range(10))
        s.leave_window(a, window, sinks)
        s.free(a)
        assert sorted(s.free_pages) == list(range(10))


def test_compaction_moves_pages_to_the_front():
    rng = random.Random(5)
    s = Sequences(n_pages=40)
    content = {}  # page -> (sequence, index) as the copies would leave it
    s._copy = lambda src, dst: content.update({d: content[x] for x, d in zip(src, dst)})
    live = []
    for _ in range(60):
        if live and rng.random() < 0.4:
            a = live.pop(rng.randrange(len(live)))
            s.free(a)
        else:
            a = s.add()
            try:
                s.extend([a], [rng.randint(1, 300)])
            except OutOfPages:
                s.free(a)
                continue
            live.append(a)
            for i, p in enumerate(s.pages[a]):
                content[p] = (a, i)
    want = {a: [content[p] for p in s.pages[a]] for a in live}
    n = s.compact()
    assert n == sum(len(s.pages[a]) for a in live) and max(p for a in live for p in s.pages[a]) == n - 1
    assert {a: [content[p] for p in s.pages[a]] for a in live} == want
    for a in live:
        assert want[a] == [(a, i) for i in range(len(s.pages[a]))]
    consistent(s)


def test_cache_tensors_are_checked():
    k, v = torch.empty(3, 2, 64, 128, dtype=torch.float8_e4m3fn), torch.empty(3, 2, 128, 64, dtype=torch.float8_e4m3fn)
    s = torch.empty(3, 2)
    KVCache(k, v, s, s.clone())
    for bad in ((k, k, s, s), (k.view(torch.uint8), v, s, s), (k, v, s.double(), s), (k, v, s, s.t()), (k[:, :, :, :96], v, s, s),
                (torch.empty(3, 2, 64, 32, dtype=torch.float8_e4m3fn), torch.empty(3, 2, 32, 64, dtype=torch.float8_e4m3fn), s, s)):
        with pytest.raises(ValueError):
            KVCache(*bad)
    cache = KVCache.empty(3, 2, 64, "cpu")
    i = torch.zeros(2, dtype=torch.int32)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # not on a device
        B.ca_cache_append(cache, x, x, i, i[:1], i[None])


def test_calls_refuse_on_the_host():
    L = B.lib()
    fake = 1 << 20
    good = dict(n_pages=4, n_kv_heads=2, head_dim=64, k=fake, v=fake, k_scale=fake, v_scale=fake)
    batch = dict(n_seqs=2, table_width=3, total_rows=4, q_start=fake, kv_len=fake, page_table=fake)
    ref = lambda cls, d: ctypes.byref(cls(**d))  # noqa: E731

    def attend(c=good, b=batch, hq=4, window=0, sinks=0, q=fake, o=fake, ws=fake, n=1 << 40):
        return L.ca_cache_attend(ref(CacheDesc, c), ref(B.CacheBatch, b), hq, 0.0, window, sinks, q, o, None, ws, n, None)

    arg, uns = B.CA_ERR_INVALID_ARG, B.CA_ERR_UNSUPPORTED
    for change, code in ((dict(n_pages=-1), arg), (dict(n_kv_heads=0), arg), (dict(n_kv_heads=2000), uns), (dict(head_dim=96), uns),
                         (dict(k=None), arg), (dict(v_scale=None), arg), (dict(k=fake + 8), arg)):
        c = good | change
        assert attend(c=c) == code
        assert L.ca_cache_append(ref(CacheDesc, c), ref(B.CacheBatch, batch), fake, fake, None) == code
        assert L.ca_cache_copy_pages(ref(CacheDesc, c), fake, fake, 1, None) == code
        assert L.ca_cache_attend_workspace_bytes(ref(CacheDesc, c), 4, ctypes.byref(ctypes.c_size_t())) == code
    for change, code in ((dict(n_seqs=-1), arg), (dict(total_rows=-1), arg), (dict(table_width=-1), arg), (dict(n_seqs=4097), uns),
                         (dict(table_width=1 << 24), uns), (dict(total_rows=1 << 30), uns), (dict(q_start=None), arg), (dict(kv_len=None), arg),
                         (dict(page_table=None), arg)):
        b = batch | change
        assert attend(b=b) == code
        assert L.ca_cache_append(ref(CacheDesc, good), ref(B.CacheBatch, b), fake, fake, None) == code
    assert attend(b=batch | dict(total_rows=(1 << 30) - 1, table_width=1 << 22)) == uns
    assert attend(hq=3) == uns and attend(hq=0) == uns and attend(window=-1) == arg and attend(sinks=-1) == arg
    assert attend(q=None) == arg and attend(o=None) == arg
    assert attend(ws=None) == attend(n=100) == attend(ws=fake + 16) == B.CA_ERR_WORKSPACE
    assert L.ca_cache_attend(None, ref(B.CacheBatch, batch), 4, 0.0, 0, 0, fake, fake, None, fake, 1 << 40, None) == arg
    assert L.ca_cache_attend(ref(CacheDesc, good), None, 4, 0.0, 0, 0, fake, fake, None, fake, 1 << 40, None) == arg
    assert L.ca_cache_append(ref(CacheDesc, good), ref(B.CacheBatch, batch), None, fake, None) == arg
    assert L.ca_cache_copy_pages(ref(CacheDesc, good), fake, fake, -1, None) == arg
    assert L.ca_cache_copy_pages(ref(CacheDesc, good), None, fake, 1, None) == arg
    assert L.ca_cache_attend_workspace_bytes(ref(CacheDesc, good), 3, ctypes.byref(ctypes.c_size_t())) == uns
    assert L.ca_cache_attend_workspace_bytes(ref(CacheDesc, good), 4, None) == arg
    # nothing to do: no launch, no error
    for b in (batch | dict(n_seqs=0), batch | dict(total_rows=0)):
        assert attend(b=b, q=None, o=None, ws=None) == B.CA_OK
        assert L.ca_cache_append(ref(CacheDesc, good), ref(B.CacheBatch, b), None, None, None) == B.CA_OK
    assert L.ca_cache_copy_pages(ref(CacheDesc, good), None, None, 0, None) == B.CA_OK


def test_refusals_of_rows_out_of_line_and_of_more_work_than_a_launch_holds():
    """Bytes that are read 16 at a time lie on multiples of 16; a launch has less than 2^24 workgroups."""
    L, fake, arg, uns = B.lib(), 1 << 20, B.CA_ERR_INVALID_ARG, B.CA_ERR_UNSUPPORTED
    cache = ctypes.byref(CacheDesc(4, 1024, 128, fake, fake, fake, fake))
    small = ctypes.byref(CacheDesc(4, 1, 64, fake, fake, fake, fake))
    batch = ctypes.byref(B.CacheBatch(2, 3, 4, fake, fake, fake))
    large = ctypes.byref(B.CacheBatch(2, 3, 1 << 22, fake, fake, fake))
    for off in (2, 8):
        assert L.ca_cache_append(cache, batch, fake + off, fake, None) == L.ca_cache_append(cache, batch, fake, fake + off, None) == arg
        for q, o in ((fake + off, fake), (fake, fake + off)):
            assert L.ca_cache_attend(cache, batch, 1024, 0.0, 0, 0, q, o, None, fake, 1 << 40, None) == arg
    assert L.ca_cache_append(cache, large, fake, fake, None) == uns
    for n in (1 << 23, 1 << 40, (1 << 63) - 1):
        assert L.ca_cache_copy_pages(small, fake, fake, n, None) == uns
    assert L.ca_cache_copy_pages(cache, fake, fake, 1 << 14, None) == uns


def test_a_window_that_is_none_is_refused():
    s = Sequences(n_pages=4)
    a = s.add()
    s.extend([a], [200])
    for window, sinks in ((0, 0), (-5, 0), (64, -1)):
        with pytest.raises(ValueError):
            s.leave_window(a, window, sinks)
    with pytest.raises(TypeError):
        s.leave_window(a, 64.0)
    assert s.pages[a] == [0, 1, 2, 3]
