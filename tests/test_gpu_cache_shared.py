"""Attention of groups of sequences that share their first pages, against the definition in 64 bits over each sequence by itself."""
import numpy as np
import pytest
import torch

import cache_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import rotary as R
from paper_2510_18121_amd.cache import KVCache, Sequences
from test_gpu_cache import DEV, filled, i32, poison, queries

pytestmark = pytest.mark.gpu


def layout(groups, lens, seed=0):
    """A page table in which the sequences of each (members, pages) have their first pages in common, and how many pages there are."""
    need = [-(-x // 64) for x in lens]
    total = sum(need) - sum(max(0, m - 1) * p for m, p in groups) + 3
    ids = list(np.random.default_rng(seed).permutation(total))
    table, s = np.full((len(lens), max(need + [1])), -1, np.int32), 0
    for m, p in groups:
        first, ids = ids[:p if m else 0], ids[p if m else 0:]
        for i in range(s, s + m):
            table[i, :p] = first
            table[i, p:need[i]], ids = ids[:need[i] - p], ids[need[i] - p:]
        s += m
    for i in range(s, len(lens)):
        table[i, :need[i]], ids = ids[:need[i]], ids[need[i]:]
    return table, total


def attend(c, q, n, lens, table, groups, lse=True, ws_rows=None, scale=0.0, arrays=None):
    start, pages = arrays or (np.concatenate([[0], np.cumsum([m for m, _ in groups])]), [p for _, p in groups])
    o = torch.full_like(q, 9.0)
    out = torch.full((q.shape[1], q.shape[0]), 9.0, device=DEV) if lse else None
    ws = B.alloc_shared_workspace(c, q.shape[1], ws_rows or q.shape[0]).fill_(0xFF)  # NaN wherever something is read first
    B.ca_cache_attend_shared(c, q, o, out, i32(np.concatenate([[0], np.cumsum(n)])), i32(lens), i32(table), i32(start), i32(pages), ws, softmax_scale=scale)
    return o, out


def run(groups, n, tails, hq, hkv, d, seed=1, **kw):
    prefix = [p for m, p in groups for _ in range(m)]
    prefix += [0] * (len(n) - len(prefix))
    lens = [64 * p + t for p, t in zip(prefix, tails)]
    table, pages = layout(groups, lens, seed)
    c = filled(pages, hkv, d)
    poison(c, lens, table)
    q = queries(sum(n), hq, d)
    got = attend(c, q, n, lens, table, groups, **kw)
    U.check(*got, U.attend(c, q, n, lens, table, scale=kw.get("scale") or None))
    return c, q, lens, table, got


HEADS = [(4, 2, 64), (8, 1, 128), (6, 2, 128), (3, 3, 64), (32, 1, 64), (40, 2, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("groups,n,tails", [
    ([(3, 1)], [1, 1, 1], [1, 64, 65]),
    ([(2, 3), (1, 5), (4, 2), (2, 0)], [1] * 9, [5, 130, 64, 1, 2, 63, 700, 100, 1]),
    ([(5, 30)], [1] * 5, [10, 1, 64, 1300, 200]),       # cut prefix, a cut tail
    ([(2, 20), (3, 17)], [3, 0, 2, 9, 1], [50, 7, 2, 9, 1100]),
    ([(2, 2), (2, 19)], [40, 64, 1, 100], [40, 300, 1, 1200]),
    ([(0, 4), (2, 1), (0, 0)], [1, 1, 1], [3, 70, 500])])  # empty groups, a sequence of none
def test_groups_of_every_kind(hq, hkv, d, groups, n, tails):
    run(groups, n, tails, hq, hkv, d)


@pytest.mark.parametrize("seqs", [16, 64, 65, 300])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (8, 1, 128)])
def test_many_sequences_of_one_group(seqs, hq, hkv, d):
    rng = np.random.default_rng(seqs)
    run([(seqs, 25)], [1] * seqs, rng.integers(1, 200, seqs).tolist(), hq, hkv, d)


@pytest.mark.parametrize("members,count", [(2, 33), (3, 70), (1, 80)])
def test_many_groups(members, count):
    rng = np.random.default_rng(members)
    groups = [(members, int(p)) for p in rng.integers(0, 22, count)]
    run(groups, [1] * (members * count), rng.integers(1, 90, members * count).tolist(), 8, 2, 128)


def test_4096_sequences():
    rng = np.random.default_rng(1)
    run([(1000, 3), (3000, 2), (50, 1)], [1] * 4096, rng.integers(1, 70, 4096).tolist(), 2, 1, 64)


def test_2048_groups():
    rng = np.random.default_rng(2)
    run([(2, int(p)) for p in rng.integers(0, 3, 2048)], [1] * 4096, rng.integers(1, 70, 4096).tolist(), 2, 1, 64)


def test_more_kv_heads_than_workgroups_of_a_kind():
    run([(3, 6)], [1, 2, 1], [5, 70, 64], 300, 300, 64)
    run([(40, 5)], [1] * 40, [5 + i for i in range(40)], 260, 260, 64)


def test_two_streams_with_a_workspace_each():
    """Calls that overlap in time: each as it is alone."""
    jobs = []
    for i, (groups, seqs, hq, hkv, d) in enumerate((([(40, 40)], 40, 32, 8, 128), ([(5, 30), (6, 50)], 11, 16, 16, 64))):
        lens = [64 * p + 100 + 7 * j for j, p in enumerate([p for m, p in groups for _ in range(m)])]
        table, pages = layout(groups, lens, seed=i)
        c, q = filled(pages, hkv, d, seed=i), queries(seqs, hq, d, seed=i)
        where = [i32(x) for x in (np.arange(seqs + 1), lens, table, np.concatenate([[0], np.cumsum([m for m, _ in groups])]), [p for _, p in groups])]
        jobs.append((c, q, where, B.alloc_shared_workspace(c, hq, seqs), torch.cuda.Stream()))
    torch.cuda.synchronize()
    alone = []
    for c, q, where, ws, _ in jobs:
        o = torch.empty_like(q)
        B.ca_cache_attend_shared(c, q, o, None, *where, ws)
        torch.cuda.synchronize()
        alone.append(o)
    outs = [[torch.empty_like(q) for _ in range(20)] for _, q, _, _, _ in jobs]
    torch.cuda.synchronize()
    for i in range(20):
        for (c, q, where, ws, stream), out in zip(jobs, outs):
            B.ca_cache_attend_shared(c, q, out[i], None, *where, ws, stream=stream)
    torch.cuda.synchronize()
    for a, out in zip(alone, outs):
        assert all(torch.equal(a, o) for o in out)


def test_tails_beyond_the_last_cache():
    """Tails of 600 MB, whose codes pass the caches by, against attention without sharing: each is off by at most 2^-8 of what the probabilities and values
    weigh, which for values of unlike signs is more than the result's own norm, so that twice 2^-8 of that bounds no less than what the two differ by here."""
    groups, tails = [(30, 20), (10, 5)], [6400 + 37 * i for i in range(40)]
    lens = [64 * p + t for (p, t) in zip([20] * 30 + [5] * 10, tails)]
    table, pages = layout(groups, lens)
    c = filled(pages, 8, 128)
    q = queries(40, 32, 128)
    o, lse = attend(c, q, [1] * 40, lens, table, groups)
    want, want_lse = torch.empty_like(q), torch.empty_like(lse)
    B.ca_cache_attend(c, q, want, want_lse, i32(np.arange(41)), i32(lens), i32(table), B.alloc_cache_workspace(c, 32))
    assert (o.double() - want.double()).norm() <= 2.0 ** -7 * want.double().norm()
    assert (lse - want_lse).abs().max() <= 2e-4


def test_groups_of_some_sequences_only():
    """Groups that begin behind the first sequence and end before the last."""
    n, lens = [1] * 6, [64 * 3 + 5, 64 * 20 + 9, 64 * 20 + 64, 64 * 20 + 1, 30, 64 * 18]
    table, pages = layout([(1, 0), (3, 20)], lens)
    c = filled(pages, 2, 128)
    poison(c, lens, table)
    q = queries(6, 8, 128)
    U.check(*attend(c, q, n, lens, table, None, arrays=([1, 4], [20])), U.attend(c, q, n, lens, table))


def test_rows_inside_the_prefix():
    """Sequences of which a row does not see all of the shared pages are attended by themselves, the others of their group are not."""
    n, lens = [70, 1, 5, 64], [64 * 4 + 60, 64 * 4 + 60, 64 * 4 + 4, 64 * 4 + 64]
    table, pages = layout([(4, 4)], lens)
    c = filled(pages, 2, 64)
    poison(c, lens, table)
    q = queries(sum(n), 4, 64)
    U.check(*attend(c, q, n, lens, table, [(4, 4)]), U.attend(c, q, n, lens, table))
    # a whole page short: no sequence has all of the group's pages
    U.check(*attend(c, q, n, lens, table, None, arrays=([0, 4], [5])), U.attend(c, q, n, lens, table))


def test_arrays_out_of_range_share_nothing_that_is_not_there():
    n, lens = [1] * 3, [64 * 2 + 5, 64 * 2 + 9, 64 * 2 + 64]
    table, pages = layout([(3, 2)], lens)
    c = filled(pages, 2, 128)
    poison(c, lens, table)
    q, want = queries(3, 8, 128), U.attend(c, queries(3, 8, 128), n, lens, table)
    for start, shared in (([0, 3], [-7]), ([0, 3], [2 ** 31 - 1]), ([-4, 3], [2]), ([0, 99], [2]), ([3, 3], [2]), ([0, 0], [2]), ([0, 0, 3, 3], [9, 2, 2])):
        U.check(*attend(c, q, n, lens, table, None, arrays=(start, shared)), want)


def test_no_groups_at_all():
    n, lens = [1, 3, 1], [1300, 70, 64]
    table, pages = layout([], lens)
    c = filled(pages, 2, 128)
    q = queries(5, 8, 128)
    U.check(*attend(c, q, n, lens, table, []), U.attend(c, q, n, lens, table))


def test_missing_pages_of_a_prefix():
    n, lens = [1] * 4, [64 * 20 + 5, 64 * 20 + 9, 64 * 20 + 64, 64 * 20 + 1]
    table, pages = layout([(4, 20)], lens)
    table[:, 3], table[:, 17], table[2, 20] = -1, pages + 9, -1
    c = filled(pages, 2, 128)
    q = queries(4, 8, 128)
    U.check(*attend(c, q, n, lens, table, [(4, 20)]), U.attend(c, q, n, lens, table))
    table[:, :20] = -1  # nobody sees anything of the prefix; one of them nothing at all
    got = attend(c, q, n, lens, table, [(4, 20)])
    U.check(*got, U.attend(c, q, n, lens, table))
    assert (got[0][2] == 0).all() and torch.isinf(got[1][:, 2]).all()


def test_rows_of_no_sequence_and_no_lse():
    c, q, lens, table, _ = run([(3, 18)], [1] * 3, [5, 6, 7], 8, 2, 128)
    more = torch.cat([q, q[:2]])
    o = torch.full_like(more, 5.0)
    ws = B.alloc_shared_workspace(c, 8, 50)
    B.ca_cache_attend_shared(c, more, o, None, i32([0, 1, 2, 3]), i32(lens), i32(table), i32([0, 3]), i32([18]), ws)
    U.check(o[:3], None, U.attend(c, q, [1] * 3, lens, table))
    assert (o[3:] == 5).all()


@pytest.mark.parametrize("scale", [0.02, 0.7])
def test_softmax_scale(scale):
    run([(4, 18)], [1] * 4, [5, 6, 700, 64], 8, 2, 128, scale=scale)


def test_scores_far_apart():
    """The prefix holds all of a row's weight, or none of it."""
    n, lens = [1] * 3, [64 * 17 + 5, 64 * 17 + 70, 64 * 17 + 64]
    table, pages = layout([(3, 17)], lens)
    c = filled(pages, 1, 128)
    for ids, f in ((table[0, :17], 30.0), (table[0, 17:], 1.0)):
        for p in ids[ids >= 0].tolist():
            c.k_scale[p] *= f
    q = queries(3, 8, 128)
    U.check(*attend(c, q, n, lens, table, [(3, 17)]), U.attend(c, q, n, lens, table))
    for p in table[:, 17:][table[:, 17:] >= 0].tolist():
        c.k_scale[p] *= 900.0
    U.check(*attend(c, q, n, lens, table, [(3, 17)]), U.attend(c, q, n, lens, table))


def test_graph_follows_the_arrays_and_streams():
    """Captured once; lengths, pages and groups change between replays.  The same bits each time, and on another stream."""
    rng = np.random.default_rng(3)
    n, most = [1] * 12, [64 * 40] * 12
    c = filled(500, 2, 128)
    q = queries(12, 8, 128)
    start, lens, table = i32(np.arange(13)), i32(most), i32(np.zeros((12, 40)))
    group_start, pages = i32([0, 4, 12]), i32([1, 1])
    o, lse, ws = torch.zeros_like(q), torch.zeros(8, 12, device=DEV), B.alloc_shared_workspace(c, 8, 12)
    call = lambda **kw: B.ca_cache_attend_shared(c, q, o, lse, start, lens, table, group_start, pages, ws, **kw)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for groups in ([(4, 20), (8, 30)], [(10, 3), (2, 33)], [(0, 1), (12, 18)]):
        tails = rng.integers(1, 64 * 5, 12).tolist()
        lengths = [64 * p + t for (m, p) in groups for t in [tails.pop() for _ in range(m)]]
        t, _ = layout(groups, lengths, seed=len(groups))
        wide = np.full((12, 40), -1, np.int32)
        wide[:, :t.shape[1]] = t
        q.copy_(queries(12, 8, 128, seed=int(t.sum()) % 1000))
        lens.copy_(i32(lengths)), table.copy_(i32(wide)), group_start.copy_(i32([0, groups[0][0], 12])), pages.copy_(i32([p for _, p in groups]))
        ws.fill_(0xFF), o.fill_(5.0), lse.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        U.check(o, lse, U.attend(c, q, n, lengths, wide))
        before = o.clone(), lse.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, before[0]) and torch.equal(lse, before[1])
        o.fill_(5.0)
        torch.cuda.synchronize()
        call(stream=side)
        side.synchronize()
        assert torch.equal(o, before[0]) and torch.equal(lse, before[1])


def test_answers_to_one_prompt():
    """As a server uses it all: a prompt's keys turned and appended, forked, drafts of unlike lengths behind it, token by token."""
    hq, hkv, d = 8, 2, 128
    cache = KVCache.empty(200, hkv, d, DEV)
    s, r = Sequences([cache]), R.Rotation(d, base=5e5, device=DEV)
    gain = 1 + 0.2 * torch.randn(d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4))
    prompt = s.add()
    where = s.extend([prompt], [1500])
    k = queries(1500, hkv, d)
    B.ca_rotate(r, k, None, k, None, where=where, q_gain=gain)
    B.ca_cache_append(cache, k, queries(1500, hkv, d, seed=1), *where)
    forks = [s.fork(prompt) for _ in range(7)]
    other = s.add()
    batch, ws = [*forks[:4], *forks[4:], other], B.alloc_shared_workspace(cache, hq, 200)
    for step, rows in enumerate(([1] * 8, [5, 1, 2, 1, 60, 1, 1, 3], [1] * 8)):
        where = s.extend(batch, rows)
        groups = s.groups(batch, rows)
        assert groups[1].tolist()[0] == 1500 // 64
        q, k, v = (queries(sum(rows), h, d, seed=10 * step + i) for i, h in enumerate((hq, hkv, hkv)))
        B.ca_rotate(r, q, k, q, k, where=where, q_gain=gain, k_gain=gain)
        B.ca_cache_append(cache, k, v, *where)
        o, lse = torch.empty_like(q), torch.empty(hq, q.shape[0], device=DEV)
        B.ca_cache_attend_shared(cache, q, o, lse, *where, *groups, ws)
        want = U.attend(cache, q, rows, where[1].tolist(), where[2].cpu().numpy())
        U.check(o, lse, want)
        B.ca_cache_attend(cache, q, o, lse, *where, B.alloc_cache_workspace(cache, hq))
        U.check(o, lse, want)


def test_tensors_that_are_refused():
    c = filled(10, 2, 64)
    q = queries(2, 4, 64)
    o, ws, args = torch.empty_like(q), B.alloc_shared_workspace(c, 4, 2), (i32([0, 1, 2]), i32([70, 70]), i32([[0, 1], [0, 2]]))
    B.ca_cache_attend_shared(c, q, o, None, *args, i32([0, 2]), i32([1]), ws)
    for groups in ((i32([0]), i32([1])), (i32([0, 2]).long(), i32([1])), (i32([0, 2]), i32([1]).cpu())):
        with pytest.raises(ValueError):
            B.ca_cache_attend_shared(c, q, o, None, *args, *groups, ws)
    with pytest.raises(B.CaError):
        B.ca_cache_attend_shared(c, q, o, None, *args, i32([0, 2]), i32([1]), ws[:-256])
    with pytest.raises(B.CaError):
        B.ca_cache_attend_shared(c, q, o, None, *args, i32([0, 1, 2, 2]), i32([1, 1, 1]), ws)
