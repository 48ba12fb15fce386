"""Steps of a server from a captured graph: tokens appended and attended for a batch whose lengths, pages and idle places change between replays; and a pool beyond
4 GiB of codes."""
import numpy as np
import pytest
import torch

import cache_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd.cache import KVCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


@pytest.mark.parametrize("seqs", [3, 64, 65])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (16, 4, 128)])
def test_a_captured_step_follows_lengths_pages_and_idle_places(seqs, hq, hkv, d):
    rng, g = np.random.default_rng(seqs), torch.Generator(device=DEV).manual_seed(seqs)
    width, window, sinks = 24, 700, 5
    pages = seqs * width
    eager, captured = (KVCache.empty(pages, hkv, d, DEV) for _ in range(2))
    lens = rng.integers(0, 64 * width - 4, seqs)
    lens[:3] = 63, 64, 64 * width - 4
    own = rng.permutation(pages).reshape(seqs, width).astype(np.int32)
    for c in (eager, captured):  # what was there before the first step, the same in both
        for x in (c.k, c.v):
            x.copy_(torch.randn(x.shape, generator=torch.Generator(device=DEV).manual_seed(7), device=DEV).to(U.F8))
        c.k_scale.fill_(2.0 ** -8), c.v_scale.fill_(2.0 ** -8)
    k, v, q = torch.zeros(seqs, hkv, d, dtype=torch.bfloat16, device=DEV), torch.zeros(seqs, hkv, d, dtype=torch.bfloat16, device=DEV), normal(g, seqs, hq, d)
    start, length, table = i32(np.arange(seqs + 1)), i32(lens), i32(own)
    src, dst = i32([-1, -1]), i32([-1, -1])
    ws = B.alloc_cache_workspace(captured, hq)
    o, lse = torch.zeros_like(q), torch.zeros(hq, seqs, device=DEV)

    def step(c, o, lse, ws):
        B.ca_cache_copy_pages(c, src, dst)
        B.ca_cache_append(c, k, v, start, length, table)
        B.ca_cache_attend(c, q, o, lse, start, length, table, ws, window=window, sinks=sinks)

    length.zero_()  # (a step of idle places alone: it changes nothing, in the warm-up and in the capture)
    step(captured, o, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured, o, lse, ws)
    for turn in range(4):
        lens = lens + 1
        now, tab = lens.copy(), own.copy()
        if turn == 2:  # a place without a sequence
            now[seqs // 2], tab[seqs // 2] = 0, -1
        if turn == 3:  # a sequence moved to the pages of the one that has none any more
            i, j = seqs // 2, seqs - 1
            now[i], tab[i] = 0, -1
            n = -(-int(lens[j]) // 64)
            pairs = own[j, n - 1], own[i, n - 1]
            src.copy_(i32([pairs[0], -1])), dst.copy_(i32([pairs[1], -1]))
            tab[j, n - 1] = pairs[1]
        length.copy_(i32(now)), table.copy_(i32(tab))
        k.copy_(normal(g, seqs, hkv, d)), v.copy_(normal(g, seqs, hkv, d) * 2.0 ** turn), q.copy_(normal(g, seqs, hq, d))
        ws.fill_(0xFF), o.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse = torch.full_like(o, 7.0), torch.zeros_like(lse)
        step(eager, want, want_lse, B.alloc_cache_workspace(eager, hq))
        assert torch.equal(o, want) and torch.equal(lse, want_lse)
        for a, b in ((captured.k, eager.k), (captured.v, eager.v)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(captured.k_scale, eager.k_scale) and torch.equal(captured.v_scale, eager.v_scale)
        idle = now == 0
        assert not o[torch.from_numpy(idle)].any()
        some = np.flatnonzero(~idle)[[0, 1, 2, -1]] if seqs > 3 else np.flatnonzero(~idle)
        U.check(o[some], lse[:, some], U.attend(eager, q[some], [1] * len(some), now[some], tab[some], window, sinks))


def test_pages_behind_4_gib_of_codes():
    """K and V of 4.3 GiB each: pages from the first to the last are written, copied and read."""
    hq, hkv, d, pages = 16, 8, 128, 70000
    assert (pages - 400) * hkv * 64 * d > 1 << 32
    c = KVCache.empty(pages, hkv, d, DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    n, lens = [700, 1, 130], [700, 1, 130]
    ids = np.concatenate([np.arange(pages - 14, pages), [0, 32768, 65536, 65535]]).astype(np.int32)
    table = np.full((3, 11), -1, np.int32)
    table[0], table[1, 0], table[2, :3] = ids[:11], ids[11], ids[[14, 15, 16]]
    new, q = normal(g, 2, sum(n), hkv, d), normal(g, sum(n), hq, d)
    where = i32(np.concatenate([[0], np.cumsum(n)])), i32(lens), i32(table)
    B.ca_cache_append(c, new[0], new[1], *where)
    # the same tokens in a small cache, bit for bit
    small, at = KVCache.empty(18, hkv, d, DEV), {int(p): i for i, p in enumerate(ids)}
    near = np.array([[at.get(int(p), -1) for p in row] for row in table], np.int32)
    B.ca_cache_append(small, new[0], new[1], where[0], where[1], i32(near))
    far = torch.from_numpy(ids).long().to(DEV)
    used = sorted({int(p) for p in near.flatten() if p >= 0})
    for x, y in ((c.k, small.k), (c.v, small.v)):
        x, y = x.view(torch.uint8), y.view(torch.uint8)
        for i in used:
            last = lens[[0, 1, 2][int(np.argwhere(near == i)[0, 0])]] - 64 * int(np.argwhere(near == i)[0, 1])
            a, b = x[far[i]], y[i]
            if last < 64:
                a, b = (a[:, :last], b[:, :last]) if x.shape[2] == 64 else (a[:, :, :last], b[:, :, :last])
            assert torch.equal(a, b)
    assert torch.equal(c.k_scale[far[used]], small.k_scale[used]) and torch.equal(c.v_scale[far[used]], small.v_scale[used])
    out = []
    for cache, tab in ((c, where[2]), (small, i32(near))):
        o, lse = torch.empty_like(q), torch.empty(hq, sum(n), device=DEV)
        B.ca_cache_attend(cache, q, o, lse, where[0], where[1], tab, B.alloc_cache_workspace(cache, hq))
        out.append((o, lse))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    B.ca_cache_copy_pages(c, i32([pages - 14, 65536]), i32([1, pages - 1]))
    for a, b in ((pages - 14, 1), (65536, pages - 1)):
        assert torch.equal(c.k[a].view(torch.uint8), c.k[b].view(torch.uint8)) and torch.equal(c.v[a].view(torch.uint8), c.v[b].view(torch.uint8))
        assert torch.equal(c.k_scale[a], c.k_scale[b]) and torch.equal(c.v_scale[a], c.v_scale[b])
