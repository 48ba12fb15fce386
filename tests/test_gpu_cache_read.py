"""Reading a cache back, bit for bit: code * scale in fp32, rounded to bf16."""
import numpy as np
import pytest
import torch

import cache_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import workloads as W
from paper_2510_18121_amd.cache import KVCache, Sequences
from test_gpu_cache import filled, i32, poison, queries

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def stand_for(c):
    """fp32 products on the CPU: [pages, heads, 64, d]."""
    k = c.k.cpu().view(torch.uint8).view(U.F8).float() * c.k_scale.cpu()[:, :, None, None]
    v = c.v.cpu().view(torch.uint8).view(U.F8).float() * c.v_scale.cpu()[:, :, None, None]
    return k, v.transpose(2, 3)


def rows_of(c, n, lens, table):
    out = []
    for x in stand_for(c):
        rows = []
        for i, (r, t) in enumerate(zip(n, lens)):
            for p in range(t - r, t):
                page = table[i, p // 64]
                rows.append(x[page, :, p % 64] if 0 <= page < c.n_pages else torch.zeros(c.n_kv_heads, c.head_dim))
        out.append(torch.stack(rows).to(torch.bfloat16))
    return out


def read(c, n, lens, table, extra=0, which=(True, True)):
    k, v = (torch.full((sum(n) + extra, c.n_kv_heads, c.head_dim), 9.0, dtype=torch.bfloat16, device=DEV) if w else None for w in which)
    B.ca_cache_read(c, k, v, i32(np.concatenate([[0], np.cumsum(n)])), i32(lens), i32(table))
    return [None if x is None else x.cpu() for x in (k, v)]


def same(got, want):
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("heads,d", [(1, 64), (3, 64), (8, 128), (2, 128)])
@pytest.mark.parametrize("n,lens", [([1], [1]), ([1, 1, 1], [64, 65, 1000]), ([64, 3, 0, 70], [64, 130, 10, 129]), ([200, 17, 63], [200, 100, 127])])
def test_rows_of_any_place(heads, d, n, lens):
    table, pages = U.layout(lens, seed=3)
    c = filled(pages, heads, d)
    poison(c, lens, table)
    got, want = read(c, n, lens, table, extra=5), rows_of(c, n, lens, table)
    for g, w in zip(got, want):
        assert (g[-5:] == 9).all()
        same(g[:-5], w)
    for i in (0, 1):
        alone = read(c, n, lens, table, which=(i == 0, i == 1))
        assert alone[1 - i] is None
        same(alone[i], want[i])


def test_codes_of_every_kind():
    """All 256 codes in every column: normal, below the normal range, zeros of both signs, NaN."""
    for d in (64, 128):
        c = KVCache.empty(4, 1, d, DEV)
        for codes in (c.k, c.v):
            codes.view(torch.uint8).copy_((torch.arange(4 * 64 * d, device=DEV) * 37 // 64 % 256).view(codes.shape).to(torch.uint8))
        c.k_scale.copy_(torch.tensor([[2.0 ** -6], [0.3], [2.0 ** 40], [2.0 ** -100]]))
        c.v_scale.copy_(c.k_scale)
        got, want = read(c, [256], [256], np.arange(4, dtype=np.int32)[None]), rows_of(c, [256], [256], np.arange(4, dtype=np.int32)[None])
        for g, w in zip(got, want):
            nan = torch.isnan(w)
            assert nan.any() and torch.equal(torch.isnan(g), nan)
            same(g[~nan], w[~nan])


def test_missing_pages_and_lengths_out_of_range():
    table, pages = U.layout([200, 200], seed=4)
    c = filled(pages, 2, 128)
    table[0, 1], table[1, 2] = -1, pages + 5
    got, want = read(c, [200, 150], [200, 200], table), rows_of(c, [200, 150], [200, 200], table)
    for g, w in zip(got, want):
        same(g, w)
        assert (g[64:128] == 0).all()
    # tokens before the first: their rows are left; lengths beyond the table count as far as it goes
    got = read(c, [10, 5], [4, 100000], table)
    want = rows_of(c, [4, 5], [4, 256], table)
    for g, w in zip(got, want):
        assert (g[:6] == 9).all()
        same(g[6:], w)


@pytest.mark.parametrize("seqs", [64, 65, 4096])
def test_many_sequences(seqs):
    rng = np.random.default_rng(seqs)
    lens = rng.integers(1, 200 if seqs < 100 else 70, seqs)
    n = np.minimum(lens, rng.integers(0, 4, seqs))
    table, pages = U.layout(lens, seed=5)
    c = filled(pages, 1, 64)
    for g, w in zip(read(c, n.tolist(), lens, table), rows_of(c, n, lens, table)):
        same(g, w)


def test_what_is_appended_is_read():
    """Values that the codes hold come back as they are; any others within half a step of e4m3 (2^-4 of them), or of the scale's least."""
    cache = KVCache.empty(40, 4, 128, DEV)
    s = Sequences([cache])
    a, b = s.add(), s.add()
    k = torch.randint(-8, 9, (330, 4, 128), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(torch.bfloat16) / 4
    v = queries(330, 4, 128, seed=2)
    where = s.extend([a, b], [130, 200])
    B.ca_cache_append(cache, k, v, *where)
    gk, gv = torch.empty_like(k), torch.empty_like(v)
    B.ca_cache_read(cache, gk, gv, *where)
    assert torch.equal(gk, k)
    assert ((gv.float() - v.float()).abs() <= 2.0 ** -4 * v.float().abs() + 2.0 ** -10 * 2.0 ** -6).all()
    # the tail alone, of one of them
    tail = torch.empty(7, 4, 128, dtype=torch.bfloat16, device=DEV)
    B.ca_cache_read(cache, tail, None, *s.arrays([b], [7]))
    assert torch.equal(tail, k[-7:])


def test_attention_in_16_bits_over_what_is_read():
    """A chunk behind a cached context: over the cache, and as a CA-task over the keys and values that are read back."""
    cache = KVCache.empty(20, 2, 128, DEV)
    s = Sequences([cache])
    a = s.add()
    k, v, q = queries(500, 2, 128), queries(500, 2, 128, seed=1), queries(100, 8, 128, seed=2)
    B.ca_cache_append(cache, k, v, *s.extend([a], [500]))
    rows = s.arrays([a], [100])
    o, lse = torch.empty_like(q), torch.empty(8, 100, device=DEV)
    B.ca_cache_attend(cache, q, o, lse, *rows, B.alloc_cache_workspace(cache, 8))
    bk, bv = torch.empty_like(k), torch.empty_like(v)
    B.ca_cache_read(cache, bk, bv, *s.arrays([a], [500]))
    plan = B.ca_plan(W.custom([500], [(0, 400, 100)], 8, 2, 128, seed=1))
    o2, lse2 = torch.empty_like(q), torch.empty_like(lse)
    B.ca_forward(plan, q, bk, bv, o2, lse2, B.alloc_workspace(plan))
    want = U.attend(cache, q, [100], [500], rows[2].cpu().numpy())
    U.check(o, lse, want)
    U.check(o2, lse2, want)


def test_graph_follows_the_lengths_and_streams():
    table, pages = U.layout([300, 300], seed=6)
    c = filled(pages, 2, 128)
    start, lens, t = i32([0, 100, 150]), i32([300, 300]), i32(table)
    k, v = (torch.zeros(150, 2, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.ca_cache_read(c, k, v, start, lens, t, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ca_cache_read(c, k, v, start, lens, t)
    for lengths, n in (([250, 60], [100, 50]), ([120, 299], [20, 130]), ([300, 300], [100, 50])):
        lens.copy_(i32(lengths)), start.copy_(i32([0, n[0], 150]))
        k.fill_(5.0), v.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip((k, v), rows_of(c, n, lengths, table)):
            same(g.cpu(), w)


@pytest.mark.parametrize("heads,d", [(8, 128), (16, 64)])
def test_rows_beyond_the_last_cache(heads, d):
    """More than 384 MiB, which is stored past the caches: the same bits as a sequence at a time."""
    lens = [17001, 20000, 64 * 300, 13333]
    table, pages = U.layout(lens, seed=7)
    c = filled(pages, heads, d)
    t = i32(table)
    k, v = (torch.full((sum(lens) + 3, heads, d), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.ca_cache_read(c, k, v, i32(np.concatenate([[0], np.cumsum(lens)])), i32(lens), t)
    row = 0
    for i, n in enumerate(lens):
        ki, vi = (torch.empty(n, heads, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        B.ca_cache_read(c, ki, vi, i32([0, n]), i32([n]), t[i:i + 1])
        assert torch.equal(k[row:row + n], ki) and torch.equal(v[row:row + n], vi)
        row += n
    assert (k[row:] == 9).all() and (v[row:] == 9).all()


def test_pages_beyond_4_gib():
    c = KVCache.empty((1 << 32) // (8 * 64 * 128) + 9, 8, 128, DEV)
    table = np.array([[c.n_pages - 2, 1, c.n_pages - 1]], np.int32)
    for p in table[0].tolist():
        for x in (c.k, c.v):
            x[p].view(torch.uint8).copy_(torch.randint(0, 127, x[p].shape, device=DEV, dtype=torch.uint8))
        c.k_scale[p], c.v_scale[p] = 0.5, 2.0
    k, v = (torch.empty(170, 8, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.ca_cache_read(c, k, v, i32([0, 170]), i32([170]), i32(table))
    ids = torch.as_tensor(table[0]).long().to(DEV)
    wk = (torch.stack([c.k[i].float() for i in ids.tolist()]) * 0.5).transpose(1, 2).reshape(-1, 8, 128)[:170].to(torch.bfloat16)
    wv = (torch.stack([c.v[i].float() for i in ids.tolist()]) * 2.0).permute(0, 3, 1, 2).reshape(-1, 8, 128)[:170].to(torch.bfloat16)
    assert torch.equal(k, wk) and torch.equal(v, wv)
