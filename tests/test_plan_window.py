"""Windowed plans on the host: every (row, visible key) lies in exactly one tile of its forward unit and one dK/dV unit, blocks that are
run without a mask need none, parts of cut units are disjoint and inside the workspace, and refusals."""
import ctypes

import numpy as np
import pytest

import window_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import workloads as W

CASES = {
    "whole_documents": dict(lens=[300, 1, 777], tasks=[(0, 0, 300), (1, 0, 1), (2, 0, 777)], heads=(4, 2)),
    "mha": dict(lens=[700], tasks=[(0, 0, 700)], heads=(3, 3)),
    "shards_far_apart": dict(lens=[9000, 40], tasks=[(0, 8000, 17), (0, 3, 100), (1, 10, 30), (0, 5000, 300)], heads=(8, 1)),
    "same_positions_twice": dict(lens=[500], tasks=[(0, 100, 200), (0, 150, 300)], heads=(6, 2)),
    "clipped_to_a_key_window": dict(lens=[600], tasks=[(0, 0, 300), (0, 300, 300)], heads=(4, 2), kv_lens={1: 200}),
    "single_rows": dict(lens=[5000], tasks=[(0, 4999, 1), (0, 0, 1), (0, 77, 1)], heads=(16, 2)),
}


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (17, 0), (64, 4), (100, 200), (129, 0), (1024, 1), (4000, 64)])
@pytest.mark.parametrize("name", CASES)
def test_units_cover_what_rows_see(name, window, sinks):
    c = CASES[name]
    hq, hkv = c["heads"]
    b = U.batch(c["lens"], c["tasks"], hq, hkv, 64, c.get("kv_lens"))
    plan = B.ca_plan_host(b, window=window, sinks=sinks)
    fwd, bwd, lo = plan.window_units()
    last = max(int(p + n) for p, n in zip(b.task_q_pos, b.task_q_len)) - 1
    if last < window:
        assert fwd.size == 0 and plan.info()["n_fwd_units"] > 0  # nothing is hidden: the plan without a window
        return
    rows, hi = plan.rows()
    see = U.visible(b, window, sinks)
    assert sorted(rows[rows >= 0].tolist()) == sorted(np.flatnonzero(np.isin(np.arange(b.total_q), rows)).tolist()) == list(range(b.total_q))
    # forward: which keys the unit's tiles hold, and that nothing a row sees is outside them
    done = np.zeros((hq, b.total_q), int)
    hp = plan.info()["heads_packed"]
    for slot0, kv0, n_keys, head, u_hp, key0, part, n_rows in fwd:
        assert u_hp == hp and part == -1 and key0 % 64 == 0 and 0 <= key0 < n_keys
        n_sink = min(-(-sinks // 64), key0 // 64)
        keys = np.zeros(b.total_kv, int)
        keys[kv0:kv0 + 64 * n_sink] += 1
        keys[kv0 + key0:kv0 + n_keys] += 1
        assert keys.max() == 1
        r = rows[slot0:slot0 + 256 // hp]
        assert (r[:n_rows] >= 0).all() and (r[n_rows:] < 0).all()
        assert not see[r[r >= 0]][:, keys == 0].any()
        for h in range(head, head + hp):
            done[h, r[r >= 0]] += 1
    assert (done == 1).all()
    # backward
    at = np.zeros((hkv, b.total_q, b.total_kv), np.int8)
    n_wg = plan.info()["n_bwd_workgroups"]
    followers, parts = [], []
    for i, u in enumerate(bwd):
        begin, end, full, kv_row, n_valid, pos0, head, follow, count, heads, edge, _ = u.tolist()
        assert begin <= full <= edge <= end and (end - begin) % 64 == 0 and heads == hq // hkv
        if i < n_wg:
            assert count >= 1 and head == i % hkv
            if follow < 0:
                assert count == 1
                parts.append(-1 - follow)
            elif count > 1:
                followers += range(follow, follow + count - 1)
        else:
            assert count == 0
        r = rows[begin:end]
        at[head, r[r >= 0], kv_row:kv_row + n_valid] += 1
        inner = rows[full:edge]
        assert see[inner[inner >= 0]][:, kv_row:kv_row + n_valid].all() and (n_valid == 128 or (inner < 0).all())
    assert sorted(followers) == list(range(n_wg, len(bwd))) and sorted(parts) == list(range(len(parts)))
    assert at.max() <= 1 and not (see[None] & (at == 0)).any()
    combine = plan.pieces()["bwd_combine"]
    assert combine[:, 1].sum() == len(parts)
    assert plan.workspace_bytes()[1] >= len(parts) * 256 * 64 * 4 and plan.workspace_bytes() == plan.workspace_bytes_split()


def test_every_resident_key_has_a_unit():
    b = U.batch([1000], [(0, 500, 100)], 2, 1, 64)
    _, bwd, _ = B.ca_plan_host(b, window=50).window_units()
    keys = np.zeros(1000, int)
    for u in bwd:
        keys[u[3]:u[3] + u[4]] += 1
    assert (keys == 1).all()


def test_long_documents_with_sinks_are_cut():
    b = U.batch([60000], [(0, 0, 60000)], 8, 2, 128)
    plan = B.ca_plan_host(b, window=512, sinks=4)
    _, bwd, _ = plan.window_units()
    steps = (bwd[:, 1] - bwd[:, 0]) // 64 * bwd[:, 9]
    assert (bwd[:, 7] < 0).sum() > 4 and steps.max() <= 128
    assert steps[:plan.info()["n_bwd_workgroups"]].tolist() == sorted(steps[:plan.info()["n_bwd_workgroups"]], reverse=True)


def test_tiles_follow_the_window_not_the_context():
    b = U.batch([32768], [(0, 0, 32768)], 32, 8, 128)
    fwd, _, _ = B.ca_plan_host(b, window=1024).window_units()
    assert ((fwd[:, 2] - fwd[:, 5] + 63) // 64).max() <= 18


def test_refusals():
    b = U.batch([300], [(0, 0, 300)], 2, 1, 64)
    for window, sinks in ((0, 0), (-1, 0), (5, -1)):
        with pytest.raises(B.CaError) as e:
            B.ca_plan_host(b, window=window, sinks=sinks)
        assert e.value.code == B.CA_ERR_INVALID_ARG
    for window, sinks in ((1.5, 0), (8, 0.5), ("8", 0)):
        with pytest.raises(TypeError):
            B.ca_plan_host(b, window=window, sinks=sinks)
    keep = []
    d = B.make_desc(b, keep)
    assert B.lib().ca_plan_window_host(ctypes.byref(d), 5, 0, None) == B.CA_ERR_INVALID_ARG
    assert B.lib().ca_plan_window_host(None, 5, 0, ctypes.byref(ctypes.c_void_p())) == B.CA_ERR_INVALID_ARG
    assert B.lib().ca_plan_window_units(None, 0, None) == 0
    b.task_kv_len[0] = 0
    with pytest.raises(B.CaError):
        B.ca_plan_host(b, window=5)


def test_a_window_that_hides_nothing_gives_the_plan_without_one():
    b = W.config(1)
    a, c = B.ca_plan_host(b), B.ca_plan_host(b, window=1 << 40, sinks=7)
    assert a.info() == c.info() and (a.fwd_units() == c.fwd_units()).all() and (a.bwd_units() == c.bwd_units()).all()
    assert [x.size for x in c.window_units()] == [0, 0, 0]


def test_positions_far_beyond_the_keys():
    """A clipped task may sit at positions beyond 32 bits: its rows see the sinks, or nothing."""
    b = U.batch([100], [(0, 0, 100)], 2, 1, 64)
    b.task_q_pos[0] = 1 << 40
    plan = B.ca_plan_host(b, window=1000, sinks=3)
    _, _, lo = plan.window_units()
    assert set(lo.tolist()) == {100}


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (30, 7), (30, 100)])
def test_no_unit_spans_keys_between_its_windows_that_nobody_sees(window, sinks):
    """From the first key of its windows on, a unit's keys are all seen by some row of it: tasks a few positions apart, whose keys end early or not."""
    for gap in (0, 1, 2, 40, 63, 64):
        at = [200 + (10 + window - 1 + gap) * i for i in range(6)]
        b = U.batch([900], [(0, p, 10) for p in at], 4, 1, 64, {2: at[2] - window + 2, 4: at[4] + 5})
        plan = B.ca_plan_host(b, window=window, sinks=sinks)
        fwd, _, lo = plan.window_units()
        rows, hi = plan.rows()
        for slot0, _, n_keys, _, hp, key0, _, n in fwd:
            seen = np.zeros(n_keys + 1, bool)
            for s in range(slot0, slot0 + n):
                seen[lo[s]:hi[s] + 1] = True
            first = np.flatnonzero(seen)
            assert len(first) == 0 or (seen[first[0]:first[-1] + 1].all() and key0 == first[0] // 64 * 64)
            assert len(first) == 0 or first[-1] == n_keys - 1 or not seen[n_keys - 1:].any()
