"""The cache in 8 bits on the GPU: appending bit for bit, attention against its definition in 64 bits, copies, and all of them together."""
import numpy as np
import pytest
import torch

import cache_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd.cache import KVCache, Sequences

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def filled(pages, heads, d, seed=0):
    """A cache in use, each (page, head) with scales of its own; page 0 .. are random, nothing is NaN yet."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    c = KVCache.empty(pages, heads, d, DEV)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x = torch.randn(codes.shape, generator=g, device=DEV)
        x *= torch.exp2(torch.randint(-2, 2, (pages, heads, 1, 1), generator=g, device=DEV).float())
        scale.copy_(x.abs().amax((2, 3)) / 448 * 1.1)
        codes.copy_((x / scale[:, :, None, None]).to(U.F8))
    return c


def poison(c, lens, table):
    """NaN codes and scales wherever no token of a sequence is."""
    used = np.zeros(c.n_pages, bool)
    k, v = c.k.view(torch.uint8), c.v.view(torch.uint8)
    for i, n in enumerate(lens):
        ids = table[i, :-(-n // 64)]
        used[ids[(ids >= 0) & (ids < c.n_pages)]] = True
        if n % 64 and ids[-1] >= 0:
            k[int(ids[-1]), :, n % 64:] = 0x7F
            v[int(ids[-1]), :, :, n % 64:] = 0xFF
    for p in np.flatnonzero(~used):
        k[int(p)], v[int(p)], c.k_scale[int(p)], c.v_scale[int(p)] = 0x7F, 0x7F, float("nan"), float("nan")


def queries(rows, hq, d, seed=0):
    return torch.randn(rows, hq, d, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(torch.bfloat16)


def attend(c, q, n, lens, table, window=None, sinks=0, **kw):
    o = torch.full_like(q, 9.0)
    lse = torch.full((q.shape[1], q.shape[0]), 9.0, device=DEV)
    ws = B.alloc_cache_workspace(c, q.shape[1]).fill_(0xFF)  # NaN wherever something is read first
    B.ca_cache_attend(c, q, o, lse, i32(np.concatenate([[0], np.cumsum(n)])), i32(lens), i32(table), ws, window=window, sinks=sinks, **kw)
    return o, lse


HEADS = [(4, 2, 64), (8, 1, 128), (6, 2, 128), (3, 3, 64), (32, 1, 64), (40, 2, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("window,sinks", [(None, 0), (1, 0), (100, 0), (64, 3), (700, 130)])
def test_single_tokens(hq, hkv, d, window, sinks):
    lens = [1, 63, 64, 65, 1000, 129, 2, 1731]
    table, pages = U.layout(lens, seed=1)
    c = filled(pages, hkv, d)
    poison(c, lens, table)
    q, n = queries(len(lens), hq, d), [1] * len(lens)
    U.check(*attend(c, q, n, lens, table, window, sinks), U.attend(c, q, n, lens, table, window, sinks))


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("window,sinks", [(None, 0), (1, 1), (130, 0), (64, 70)])
def test_chunks(hq, hkv, d, window, sinks):
    n, lens = [5, 0, 64, 1, 200], [300, 50, 64, 777, 261]
    table, pages = U.layout(lens, seed=2)
    c = filled(pages, hkv, d)
    poison(c, lens, table)
    q = queries(sum(n), hq, d)
    U.check(*attend(c, q, n, lens, table, window, sinks), U.attend(c, q, n, lens, table, window, sinks))


@pytest.mark.parametrize("n", [[1], [3], [40]])
@pytest.mark.parametrize("d", [64, 128])
def test_long_sequences_are_split(n, d):
    lens = [70001]
    table, pages = U.layout(lens, seed=3)
    c = filled(pages, 2, d)
    poison(c, lens, table)
    q = queries(n[0], 4, d)
    U.check(*attend(c, q, n, lens, table), U.attend(c, q, n, lens, table))


def test_a_long_sequence_among_many_short_ones():
    rng = np.random.default_rng(4)
    lens = rng.integers(1, 300, 300).tolist()
    lens[17], lens[18], lens[250] = 20000, 1, 9000
    table, pages = U.layout(lens, seed=4)
    c = filled(pages, 1, 64)
    poison(c, lens, table)
    q, n = queries(len(lens), 2, 64), [1] * len(lens)
    U.check(*attend(c, q, n, lens, table), U.attend(c, q, n, lens, table))


def test_rows_that_see_nothing_rows_of_no_sequence_and_missing_pages():
    n, lens = [1, 2, 1, 3, 2], [0, 130, 200, 2, 500]  # (a sequence without tokens, and one with fewer tokens than rows)
    table, pages = U.layout(lens, seed=5)
    table[1, 1], table[1, 0], table[4, 2] = -1, pages + 7, -5
    table[2] = -1
    c = filled(pages, 2, 64)
    poison(c, [0, 130, 0, 2, 500], table)
    q = queries(sum(n) + 4, 4, 64)
    o, lse = attend(c, q, n, lens, table)
    assert (o[-4:] == 9).all() and (lse[:, -4:] == 9).all()  # rows behind the last sequence
    got_o, got_lse = o.double().cpu(), lse.double().cpu()
    assert (got_o[0] == 0).all() and (got_lse[:, 0] == -np.inf).all()          # no token
    assert (got_o[3] == 0).all() and (got_lse[:, 3] == -np.inf).all()          # no page
    assert (got_o[4] == 0).all() and (got_lse[:, 4] == -np.inf).all()          # a row before the first token
    # the third page of sequence 1 is there: its last two rows see tokens 128 and 129
    U.check(o[1:3], lse[:, 1:3], U.attend(c, q[1:3], [2], [130], table[1:2]))
    U.check(o[5:7], lse[:, 5:7], U.attend(c, q[5:7], [2], [2], table[3:4]))
    U.check(o[7:9], lse[:, 7:9], U.attend(c, q[7:9], [2], [500], table[4:5]))


def test_values_out_of_range_stay_inside_the_tensors():
    """Starts beyond the rows, lengths beyond the table: what is there counts."""
    lens = [100, 64]
    table, pages = U.layout(lens, seed=6)
    c = filled(pages, 2, 64)
    q = queries(3, 4, 64)
    o, lse = torch.full_like(q, 9.0), torch.full((4, 3), 9.0, device=DEV)
    ws = B.alloc_cache_workspace(c, 4)
    B.ca_cache_attend(c, q, o, lse, i32([0, 2, 1 << 30]), i32([100, 1 << 30]), i32(table), ws)
    U.check(o, lse, U.attend(c, q, [2, 1], [100, 128], table))
    B.ca_cache_attend(c, q, o, lse, i32([-5, 1, 0]), i32([-100, 3]), i32(table), ws)  # descending: nobody's rows
    assert (o[0] == 0).all() and (lse[:, 0] == -np.inf).all()


def test_scores_that_grow_along_the_pages_and_a_softmax_scale():
    lens = [900]
    table, pages = U.layout(lens, seed=7)
    c = filled(pages, 1, 128)
    for i, p in enumerate(table[0].tolist()):
        c.k_scale[p] *= 0.05 * 1.5 ** i
    q = queries(1, 8, 128)
    U.check(*attend(c, q, [1], lens, table, softmax_scale=0.3), U.attend(c, q, [1], lens, table, scale=0.3))


@pytest.mark.parametrize("rows", [1, 20, 200])
def test_scales_far_from_one(rows):
    """V's of 0, tiny, huge and not a power of two, beside each other; a K scale of 0."""
    lens = [600]
    table, pages = U.layout(lens, seed=21)
    c = filled(pages, 2, 64)
    for i, p in enumerate(table[0].tolist()):
        c.v_scale[p] = (0.3, 0.0, 2.0 ** -60, 1e-3, 2.0 ** -120, 0.7, 1.0, 2.0 ** -39, 3.0, 0.5)[i]
        if i == 3:
            c.k_scale[p] = 0.0
    q = queries(rows, 4, 64)
    U.check(*attend(c, q, [rows], lens, table), U.attend(c, q, [rows], lens, table))
    c.v_scale *= 2.0 ** 50
    o, lse = attend(c, q, [rows], lens, table)
    want = U.attend(c, q, [rows], lens, table)
    U.check(o, lse, want)


@pytest.mark.parametrize("seqs,hq,hkv,d", [(70, 16, 8, 128), (70, 16, 8, 64), (520, 4, 1, 64), (1100, 1, 1, 128)])
@pytest.mark.parametrize("rows", [1, 6, 20])
@pytest.mark.parametrize("window,sinks", [(None, 0), (90, 5)])
def test_more_tiles_than_the_chip_has_room_for(seqs, hq, hkv, d, rows, window, sinks):
    """Two and more tiles per CU, of sequences from no token to thousands, most of them short; up to 1, 6 and 20 rows of each."""
    rng = np.random.default_rng(seqs + rows)
    lens = (rng.integers(0, 260, seqs)).tolist()
    lens[3], lens[seqs - 2], lens[seqs // 2] = 5000, 2900, 0
    n = [rows] * seqs if rows == 1 else rng.integers(rows - 1, rows + 1, seqs).tolist()
    table, pages = U.layout(lens, seed=31)
    c = filled(pages, hkv, d)
    poison(c, lens, table)
    q = queries(sum(n), hq, d)
    U.check(*attend(c, q, n, lens, table, window, sinks), U.attend(c, q, n, lens, table, window, sinks))


@pytest.mark.parametrize("d,pages", [(128, 3200), (64, 6300)])
@pytest.mark.parametrize("rows", [[1] * 4, [1] * 70, [5] * 70])
def test_a_large_pool_gives_the_bits_of_a_small_one(d, pages, rows):
    """Of a pool of 400 MiB codes pass the caches by; the same tokens in a small one do not."""
    rng = np.random.default_rng(32)
    lens = rng.integers(1, 1500, len(rows)).tolist()
    lens[1] = 101000 if len(rows) == 4 else 6000
    table, n = U.layout(lens, seed=33)
    small, large = filled(n, 8, d), KVCache.empty(pages, 8, d, DEV)
    assert n * 8 * 128 * d <= 256 << 20 and large.n_pages * 8 * 128 * d > 384 << 20 and len(lens) * table.shape[1] >= large.n_pages
    ids = torch.from_numpy(rng.permutation(large.n_pages)[:n]).to(DEV)
    for x, y in ((small.k, large.k), (small.v, large.v)):
        y.view(torch.uint8).fill_(0x7F)
        y.view(torch.uint8)[ids] = x.view(torch.uint8)
    for x, y in ((small.k_scale, large.k_scale), (small.v_scale, large.v_scale)):
        y.fill_(float("nan"))
        y[ids] = x
    moved = np.where(table >= 0, ids.cpu().numpy()[np.maximum(table, 0)], -1).astype(np.int32)
    q = queries(sum(rows), 32, d)
    for window, sinks in ((None, 0), (90000, 3)):
        for a, b in zip(attend(small, q, rows, lens, table, window, sinks), attend(large, q, rows, lens, moved, window, sinks)):
            assert torch.equal(a, b)


def test_as_many_sequences_as_there_may_be():
    n, lens = [1] * 4096, (np.arange(4096) % 3 + 1).tolist()
    table, pages = U.layout(lens, seed=22)
    c = power_scales(filled(pages, 1, 64))
    new, q = new_tokens(4096, 1, 64, 23), queries(4096, 2, 64)
    want = held(c)
    U.append(want, new.double().cpu().numpy(), n, lens, table)
    do_append(c, new, n, lens, table)
    same(c, want)
    U.check(*attend(c, q, n, lens, table), U.attend(c, q, n, lens, table))
    with pytest.raises(B.CaError) as e:
        attend(c, q, n + [0], lens + [0], np.concatenate([table, table[:1]]))
    assert e.value.code == B.CA_ERR_UNSUPPORTED


@pytest.mark.parametrize("g", [3, 5, 7, 24, 64])
def test_groups_that_are_no_power_of_two_and_rows_that_cross_tiles(g):
    n, lens = [37, 90, 1], [500, 90, 33]
    table, pages = U.layout(lens, seed=24)
    c = filled(pages, 1, 64)
    poison(c, lens, table)
    q = queries(sum(n), g, 64)
    for window, sinks in ((None, 0), (50, 2)):
        U.check(*attend(c, q, n, lens, table, window, sinks), U.attend(c, q, n, lens, table, window, sinks))


def test_runs_repeat_bit_for_bit_also_from_a_graph_that_follows_the_lengths():
    lens = [5000, 700, 64]
    table, pages = U.layout([5200, 900, 200], seed=8)
    c = filled(pages, 2, 128)
    q, n = queries(3, 8, 128), [1, 1, 1]
    want = attend(c, q, n, lens, table)
    o, lse, ws = torch.zeros_like(q), torch.zeros(8, 3, device=DEV), B.alloc_cache_workspace(c, 8)
    start, length, tab = i32([0, 1, 2, 3]), i32(lens), i32(table)
    call = lambda: B.ca_cache_attend(c, q, o, lse, start, length, tab, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for more in (0, 1, 100):
        length.copy_(i32(lens) + more)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        want = attend(c, q, n, [x + more for x in lens], table)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


def test_two_streams_with_a_workspace_each():
    lens = [3000, 10]
    table, pages = U.layout(lens, seed=9)
    c = filled(pages, 2, 64)
    qs = [queries(2, 4, 64, seed=s) for s in range(2)]
    want = [attend(c, q, [1, 1], lens, table) for q in qs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in qs], []
    for q, st in zip(qs, streams):
        with torch.cuda.stream(st):
            got.append(attend(c, q, [1, 1], lens, table))
    torch.cuda.synchronize()
    for (a, b), (x, y) in zip(got, want):
        assert torch.equal(a, x) and torch.equal(b, y)


# ------------------------------------------------------------------------------------------------ append
def held(c):
    return {"k": c.k.cpu().double().numpy(), "v": c.v.cpu().double().numpy().transpose(0, 1, 3, 2).copy(), "ks": c.k_scale.cpu().double().numpy(),
            "vs": c.v_scale.cpu().double().numpy()}


def power_scales(c):
    for scale in (c.k_scale, c.v_scale):
        scale.copy_(torch.exp2(torch.ceil(torch.log2(scale))))
    return c


def new_tokens(rows, heads, d, seed, spread=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(2, rows, heads, d, generator=g, device=DEV)
    return (x * torch.exp2(spread * torch.randn(2, rows, heads, 1, generator=g, device=DEV))).to(torch.bfloat16)


def do_append(c, new, n, lens, table):
    B.ca_cache_append(c, new[0], new[1], i32(np.concatenate([[0], np.cumsum(n)])), i32(lens), i32(table))


def same(c, want):
    got = held(c)
    for name in want:
        assert np.array_equal(got[name], want[name], equal_nan=True), name


@pytest.mark.parametrize("heads,d", [(2, 64), (1, 128), (8, 128), (5, 64)])
@pytest.mark.parametrize("spread", [0.0, 3.0])
@pytest.mark.parametrize("n,lens", [([1, 1, 1, 1, 1, 1], [1, 64, 65, 100, 128, 1000]), ([300, 0, 1, 64, 63, 7], [300, 40, 70, 130, 63, 71]),
                                    ([128, 2], [128, 3]), ([1, 2] * 50, [5, 130] * 50)])
def test_append_bit_for_bit(heads, d, spread, n, lens):
    table, pages = U.layout(lens, seed=11)
    c = power_scales(filled(pages, heads, d, seed=1))
    new = new_tokens(sum(n), heads, d, 12, spread)
    want = held(c)
    U.append(want, new.double().cpu().numpy(), n, lens, table)
    do_append(c, new, n, lens, table)
    same(c, want)
    do_append(c, new, n, lens, table)  # the same tokens once more: nothing grows
    same(c, want)


def test_append_token_by_token_with_growing_magnitudes():
    c = KVCache.empty(3, 2, 64, DEV)
    for x in (c.k, c.v):
        x.view(torch.uint8).fill_(0)
    c.k_scale.fill_(float("nan")), c.v_scale.fill_(float("nan"))  # forgotten with the page's first token
    want = held(c)
    table = np.array([[2, 0]], np.int32)
    for p in range(100):
        new = new_tokens(1, 2, 64, 100 + p) * 2.0 ** (p / 7 - 5)
        U.append(want, new.double().cpu().numpy(), [1], [p + 1], table)
        do_append(c, new, [1], [p + 1], table)
    same(c, want)


def test_append_zeros_tiny_and_huge_values():
    c = KVCache.empty(6, 1, 64, DEV)
    for x in (c.k, c.v):
        x.view(torch.uint8).fill_(0x11)
    c.k_scale.fill_(1), c.v_scale.fill_(1)
    new = torch.zeros(2, 6, 1, 64, dtype=torch.bfloat16, device=DEV)
    new[:, 1] = 2.0 ** -130
    new[:, 2] = torch.finfo(torch.bfloat16).max
    new[:, 3] = -448.0
    new[:, 4] = 450.0
    new[:, 5, :, :32] = 2.0 ** -126
    table, want = np.arange(6, dtype=np.int32)[:, None], held(c)
    U.append(want, new.double().cpu().numpy(), [1] * 6, [1] * 6, table)
    do_append(c, new, [1] * 6, [1] * 6, table)
    same(c, want)
    assert c.k_scale[:, 0].log2().tolist() == [-126, -126, 120, 0, 1, -126]


def test_inf_and_nan_become_nan_and_do_not_touch_the_scale():
    c = KVCache.empty(1, 1, 64, DEV)
    new = torch.ones(2, 3, 1, 64, dtype=torch.bfloat16, device=DEV)
    new[:, 1, :, :2] = torch.tensor([float("inf"), float("nan")], device=DEV)
    do_append(c, new, [3], [3], np.array([[0]], np.int32))
    k, v = c.k[0, 0].float(), c.v[0, 0].float().t()
    for x in (k, v):
        assert torch.isnan(x[1, :2]).all() and torch.isfinite(x[1, 2:]).all() and torch.isfinite(x[[0, 2]]).all()
    assert c.k_scale[0, 0] == 2.0 ** -8 and c.v_scale[0, 0] == 2.0 ** -8


def test_append_leaves_other_pages_alone_and_skips_missing_ones():
    lens, n = [70, 20], [70, 20]
    table, pages = U.layout(lens, seed=13)
    c = power_scales(filled(pages, 2, 64, seed=2))
    new = new_tokens(90, 2, 64, 14)
    want = held(c)
    U.append(want, new.double().cpu().numpy()[:, :64], [64], [64], table[:1])
    broken = table.copy()
    broken[0, 1], broken[1, 0] = -1, pages
    do_append(c, new, n, lens, broken)
    same(c, want)


def test_more_rows_than_tokens():
    """Rows before a sequence's first token are not stored."""
    table = np.array([[1], [0]], np.int32)
    c, d = power_scales(filled(2, 2, 64, seed=4)), power_scales(filled(2, 2, 64, seed=4))
    new = new_tokens(8, 2, 64, 31)
    do_append(c, new, [5, 3], [3, 3], table)
    do_append(d, new[:, 2:].contiguous(), [3, 3], [3, 3], table)
    same(c, held(d))


def test_copies():
    c = filled(9, 3, 64, seed=3)
    before = [x.clone() for x in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale)]
    B.ca_cache_copy_pages(c, i32([1, 4, 4, 9, 2]), i32([0, 7, 8, 3, -1]))
    for x, y in zip((c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale), before):
        y[0], y[7], y[8] = y[1].clone(), y[4].clone(), y[4].clone()
        assert torch.equal(x, y)


def test_refusals():
    c = filled(4, 2, 64)
    x, q = new_tokens(3, 2, 64, 1)[0], queries(3, 4, 64)
    start, lens, table = i32([0, 3]), i32([3]), i32([[0]])
    ws = B.alloc_cache_workspace(c, 4)
    good = dict(q=q, o=torch.empty_like(q), lse=None, q_start=start, kv_len=lens, page_table=table, ws=ws)
    B.ca_cache_attend(c, **good)
    for change in (dict(q=q.float()), dict(o=q[:2]), dict(lse=torch.empty(3, 4, device=DEV)), dict(q_start=start.long()), dict(kv_len=start),
                   dict(page_table=table[0]), dict(page_table=table.cpu()), dict(window=0), dict(window=-3), dict(q=q[:, :, :32])):
        with pytest.raises(ValueError):
            B.ca_cache_attend(c, **(good | change))
    for change, code in ((dict(ws=None), B.CA_ERR_WORKSPACE), (dict(ws=ws[256:]), B.CA_ERR_WORKSPACE), (dict(sinks=-1), B.CA_ERR_INVALID_ARG),
                         (dict(q=q[:, :3].contiguous(), o=q[:, :3].contiguous()), B.CA_ERR_UNSUPPORTED)):
        with pytest.raises(B.CaError) as e:
            B.ca_cache_attend(c, **(good | change))
        assert e.value.code == code
    for k, v in ((x, x[:2]), (x.float(), x), (x[:, :1].contiguous(), x[:, :1].contiguous())):
        with pytest.raises(ValueError):
            B.ca_cache_append(c, k, v, start, lens, table)
    with pytest.raises(ValueError):
        B.ca_cache_copy_pages(c, start, lens)


# ------------------------------------------------------------------------------------------------ together
def test_prompts_tokens_forks_windows_and_compaction_together():
    """A small server: prompts in chunks, single tokens, a fork, pages that leave the window, a compaction; after every step the cache's
    attention is that of the tokens as the cache holds them, and those are within half a step of e4m3 of what was appended."""
    hq, hkv, d, window, sinks = 8, 2, 64, 150, 4
    caches = [KVCache.empty(40, hkv, d, DEV) for _ in range(2)]  # two layers
    for c in caches:
        poison(c, [], np.zeros((0, 1), np.int32))
    seqs = Sequences(caches)
    ws = B.alloc_cache_workspace(caches[0], hq)
    tokens = {}  # of a sequence: the K of its first layer, as appended
    seed = 0

    def step(ids, rows):
        nonlocal seed
        start, lens, table = seqs.extend(ids, rows)
        for c in caches:
            seed += 1
            new, q = new_tokens(sum(rows), hkv, d, seed), queries(sum(rows), hq, d, seed)
            B.ca_cache_append(c, new[0], new[1], start, lens, table)
            o, lse = torch.empty_like(q), torch.empty(hq, sum(rows), device=DEV)
            B.ca_cache_attend(c, q, o, lse, start, lens, table, ws, window=window, sinks=sinks)
            U.check(o, lse, U.attend(c, q, rows, lens.tolist(), table.cpu().numpy(), window, sinks))
            if c is caches[0]:
                for i, s in enumerate(ids):
                    a, e = start[i].item(), start[i + 1].item()
                    tokens[s] = torch.cat([tokens.get(s, new[0][:0]), new[0][a:e]])
        for s in ids:
            seqs.leave_window(s, window, sinks)

    def check_held():
        c = caches[0]
        held = U.values(c.k, c.k_scale)
        for s, x in tokens.items():
            for i, p in enumerate(seqs.pages[s]):
                if p >= 0:
                    want = x[64 * i:64 * i + 64].double().cpu().transpose(0, 1)
                    off = (held[p][:, :want.shape[1]] - want).abs()
                    # twice half a step (2^-4 of the value, or half the smallest step of the scale, 2^-10): a page whose scale grew is rounded again
                    assert (off <= 2 * torch.maximum(want.abs() * 2.0 ** -4, c.k_scale[p].double().cpu()[:, None, None] * 2.0 ** -10)).all()

    a, b = seqs.add(), seqs.add()
    step([a, b], [200, 33])
    step([a], [77])
    check_held()
    c = seqs.fork(a)
    tokens[c] = tokens[a]
    for _ in range(5):
        step([a, c, b], [1, 1, 1])
    check_held()
    seqs.free(b)
    del tokens[b]
    seqs.compact()
    check_held()
    step([c, a], [90, 1])
    check_held()
    used = {p for s in (a, c) for p in seqs.pages[s] if p >= 0}
    assert len(seqs.free_pages) == 40 - len(used)
