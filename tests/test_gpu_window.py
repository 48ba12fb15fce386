"""Attention with a sliding window and sinks on the GPU, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import window_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import workloads as W
from paper_2510_18121_amd.autograd import AttentionServer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def run(b, window, sinks, tensors, backward=True, mark=None):
    q, k, v, d_o = tensors
    plan = B.ca_plan(b, window=window, sinks=sinks)
    o = torch.full_like(q, mark if mark is not None else 7.0)
    lse = torch.full((b.n_q_heads, b.total_q), 7.0, device=DEV)
    ws = torch.full((max(*plan.workspace_bytes(), 256),), 0xFF, dtype=torch.uint8, device=DEV)  # NaN wherever something is read first
    B.ca_forward(plan, q, k, v, o, lse, ws)
    out = {"o": o, "lse": lse}
    if backward:
        out |= {"dq": torch.full_like(q, 7.0), "dk": torch.full_like(k, 7.0), "dv": torch.full_like(v, 7.0)}
        B.ca_backward(plan, q, k, v, o, d_o, lse, out["dq"], out["dk"], out["dv"], ws)
    return out


def check(b, window, sinks, got, tensors):
    q, k, v, d_o = tensors
    want, far = U.reference(b, window, sinks, q, k, v, d_o, got["o"])
    U.check(got, want, far, ("o", "dq", "dk", "dv"))
    lse = got["lse"].double().cpu()
    none = torch.isinf(want["lse"])
    assert (lse[none] == -np.inf).all()
    off = (lse - want["lse"]).abs()[~none]  # fp32 sums of products: 2^-20 of a large one
    assert (off <= 1e-4 + 2.0 ** -20 * want["lse"].abs()[~none]).all()
    rows = none[0]
    assert (got["o"].cpu()[rows] == 0).all() and (got["dq"].cpu()[rows] == 0).all()


SHAPES = {
    "documents": dict(lens=[300, 1, 777], tasks=[(0, 0, 300), (1, 0, 1), (2, 0, 777)]),
    "shards_far_apart": dict(lens=[2500, 40], tasks=[(0, 2300, 17), (0, 3, 100), (1, 10, 30), (0, 1200, 300)]),
    "same_positions_twice": dict(lens=[500], tasks=[(0, 100, 200), (0, 150, 300)]),
    "clipped": dict(lens=[600], tasks=[(0, 0, 300), (0, 300, 300)], kv_lens={1: 200}),
    "single_rows": dict(lens=[1500], tasks=[(0, 1499, 1), (0, 0, 1), (0, 77, 1)]),
}


@pytest.mark.parametrize("heads,d", [((4, 2), 64), ((4, 1), 128), ((3, 3), 128), ((8, 1), 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (17, 0), (63, 130), (64, 4), (129, 0), (400, 1)])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_definition(shape, window, sinks, heads, d):
    s = SHAPES[shape]
    b = U.batch(s["lens"], s["tasks"], *heads, d, s.get("kv_lens"), seed=3)
    tensors = W.make_tensors(b, DEV)
    check(b, window, sinks, run(b, window, sinks, tensors), tensors)


def test_windows_of_many_tiles_and_cut_sink_tiles():
    """4000 rows, windows of 1024 keys (whole tiles without a mask), a sink tile of 252 steps in pieces."""
    b = U.batch([4003], [(0, 0, 4003)], 8, 2, 128, seed=4)
    tensors = W.make_tensors(b, DEV)
    assert B.ca_plan_host(b, window=1024, sinks=4).pieces()["bwd_combine"].size > 0
    check(b, 1024, 4, run(b, 1024, 4, tensors), tensors)


@pytest.mark.parametrize("heads,d", [((16, 16), 64), ((16, 16), 128), ((8, 8), 64)])
def test_chained_units_of_many_documents(heads, d):
    """Short dK/dV units, several to a workgroup one after the other, and more workgroups than run at a time."""
    n_docs, n = 26, 650
    b = U.batch([n] * n_docs, [(i, 0, n) for i in range(n_docs)], *heads, d, seed=11)
    info = B.ca_plan_host(b, window=100, sinks=0).info()
    assert (info["n_bwd_workgroups"] < info["n_bwd_units"]) == (heads == (16, 16))  # (the other: whole units alone)
    tensors = W.make_tensors(b, DEV)
    first = run(b, 100, 0, tensors)
    one = U.batch([n], [(0, 0, n)], 2, 2, d)
    for doc, h in ((0, 0), (13, 4), (25, heads[0] - 2), (7, 2)):
        of = slice(doc * n, doc * n + n), slice(h, h + 2)
        part = {x: y[of] if x != "lse" else y[h:h + 2, of[0]] for x, y in first.items()}
        check(one, 100, 0, part, tuple(x[of] for x in tensors))
    for _ in range(3):
        again = run(b, 100, 0, tensors)
        assert all(torch.equal(again[x], first[x]) for x in first)


@pytest.mark.parametrize("factor", [8.0, 60.0])
def test_scores_that_outgrow_the_first_keys(factor):
    """Early keys are small and later ones large: the reference of the exponentials is outgrown and rows are computed again."""
    b = U.batch([700], [(0, 0, 700)], 4, 2, 64, seed=5)
    q, k, v, d_o = W.make_tensors(b, DEV)
    k = (k.float() * torch.linspace(0, factor, 700, device=DEV)[:, None, None]).to(torch.bfloat16)
    got = run(b, 200, 2, (q, k, v, d_o))
    check(b, 200, 2, got, (q, k, v, d_o))


def test_rows_of_no_task_and_keys_that_nobody_sees():
    b = U.batch([600, 100], [(0, 400, 64), (1, 0, 100)], 4, 2, 64, seed=6)
    b.total_q += 13  # rows behind the last task
    q, k, v, d_o = W.make_tensors(b, DEV)
    got = run(b, 100, 0, (q, k, v, d_o), mark=5.0)
    assert (got["o"][-13:] == 5.0).all() and (got["lse"][:, -13:] == 7.0).all() and (got["dq"][-13:] == 0).all()
    k0 = int(b.doc_kv_start[0])
    for n in ("dk", "dv"):
        assert (got[n][k0:k0 + 301] == 0).all() and (got[n][k0 + 464:k0 + 600] == 0).all()
        assert (got[n][k0 + 301:k0 + 464].abs().sum((1, 2)) > 0).all()


def test_a_window_over_everything_is_plain_attention_bit_for_bit():
    b = W.config(1)
    tensors = W.make_tensors(b, DEV)
    got, want = run(b, 1 << 33, 3, tensors), run(b, None, 0, tensors)
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_runs_repeat_bit_for_bit_and_documents_do_not_depend_on_their_shards():
    b = U.batch([900], [(0, 0, 900)], 8, 2, 128, seed=7)
    tensors = W.make_tensors(b, DEV)
    a, c = run(b, 130, 4, tensors), run(b, 130, 4, tensors)
    assert all(torch.equal(a[n], c[n]) for n in a)
    parts = W.custom([900], [(0, 0, 333), (0, 333, 1), (0, 334, 566)], 8, 2, 128, seed=7)
    d = run(parts, 130, 4, tensors)
    assert torch.equal(a["o"], d["o"]) and torch.equal(a["dq"], d["dq"]) and torch.equal(a["dk"], d["dk"])


def test_differentiable_op_and_gradients_against_differences():
    b = U.batch([150], [(0, 0, 150)], 2, 1, 64, seed=8)
    q, k, v, d_o = (x.detach().clone() for x in W.make_tensors(b, DEV))
    for x in (q, k, v):
        x.requires_grad_()
    server = AttentionServer(b, DEV, window=20, sinks=2)
    o = server(q, k, v)
    grads = torch.autograd.grad(o, (q, k, v), d_o)
    want, far = U.reference(b, 20, 2, q, k, v, d_o, o.detach())
    U.check(dict(zip(("dq", "dk", "dv"), grads)), want, far, ("dq", "dk", "dv"))
    # the definition's gradient itself, by central differences of its loss in 64 bits along one direction
    x = [t.detach().double().cpu() for t in (q, k, v)]
    gen = torch.Generator().manual_seed(0)
    step = [torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in x]
    loss = lambda e: (U.reference(b, 20, 2, *(t + e * u for t, u in zip(x, step)))[0]["o"] * d_o.double().cpu()).sum()  # noqa: E731
    exact = U.reference(b, 20, 2, *x, d_o)[0]
    slope = sum((exact[n] * u).sum() for n, u in zip(("dq", "dk", "dv"), step))
    assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - slope) <= 1e-6 * abs(slope) + 1e-6


def test_replayed_from_a_graph_with_eager_work_between():
    b = U.batch([800], [(0, 0, 800)], 8, 2, 64, seed=9)
    q, k, v, d_o = W.make_tensors(b, DEV)
    want = run(b, 100, 4, (q, k, v, d_o))
    plan = B.ca_plan(b, window=100, sinks=4)
    ws = B.alloc_workspace(plan, DEV)
    got = {n: torch.zeros_like(x) for n, x in want.items()}

    def step():
        B.ca_forward(plan, q, k, v, got["o"], got["lse"], ws)
        B.ca_backward(plan, q, k, v, got["o"], d_o, got["lse"], got["dq"], got["dk"], got["dv"], ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for x in got.values():
            x.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)
        assert torch.equal(run(b, 100, 4, (q, k, v, d_o))["dq"], want["dq"])


def test_too_small_a_workspace_is_refused():
    b = U.batch([800], [(0, 0, 800)], 8, 2, 64)
    q, k, v, d_o = W.make_tensors(b, DEV)
    plan = B.ca_plan(b, window=100, sinks=4)
    need = plan.workspace_bytes()[1]
    ws = torch.empty(need - 1, dtype=torch.uint8, device=DEV)
    lse = torch.zeros(8, 800, device=DEV)
    with pytest.raises(B.CaError) as e:
        B.ca_backward(plan, q, k, v, q, d_o, lse, torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), ws)
    assert e.value.code == B.CA_ERR_WORKSPACE


def test_on_the_librarys_own_workspace():
    b = U.batch([800], [(0, 0, 800)], 8, 2, 64, seed=9)
    q, k, v, d_o = tensors = W.make_tensors(b, DEV)
    want = run(b, 100, 4, tensors)
    plan = B.ca_plan(b, window=100, sinks=4)
    got = {n: torch.full_like(want[n], 7.0) for n in ("dq", "dk", "dv")}
    B.ca_backward_static_ws(plan, q, k, v, want["o"], d_o, want["lse"], got["dq"], got["dk"], got["dv"])
    assert all(torch.equal(got[n], want[n]) for n in got)


def test_two_streams_share_a_plan():
    b = U.batch([900], [(0, 0, 900)], 4, 2, 128, seed=10)
    tensors = [W.make_tensors(b, DEV), tuple(x.flip(0).contiguous() for x in W.make_tensors(b, DEV))]
    want = [run(b, 60, 1, x) for x in tensors]
    plan = B.ca_plan(b, window=60, sinks=1)
    torch.cuda.synchronize()
    got, streams = [], [torch.cuda.Stream() for _ in tensors]
    for (q, k, v, d_o), st in zip(tensors, streams):
        with torch.cuda.stream(st):
            x = {"o": torch.empty_like(q), "lse": torch.empty(4, 900, device=DEV), "dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v)}
            ws = B.alloc_workspace(plan, DEV)
            B.ca_forward(plan, q, k, v, x["o"], x["lse"], ws)
            B.ca_backward(plan, q, k, v, x["o"], d_o, x["lse"], x["dq"], x["dk"], x["dv"], ws)
            got.append(x)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert all(torch.equal(x[n], y[n]) for n in y)


def test_windowed_shards_with_key_windows_merge_to_the_whole():
    """Partial results of a windowed shard over two key windows of its context (positions counted from each), merged, and the gradients."""
    n, cut, window = 700, 384, 250
    whole = U.batch([n], [(0, 450, 250)], 4, 2, 64, seed=12)
    q, k, v, d_o = W.make_tensors(whole, DEV)
    # keys [0, cut) and [cut, n) as documents of their own, the shard a task on both; the first one's rows sit behind its keys
    parts = W.custom([cut, n - cut], [(0, 450, 250), (1, 450 - cut, 250)], 4, 2, 64, seed=12)
    parts.task_kv_len[0] = cut
    plan = B.ca_plan(parts, window=window)
    ws = B.alloc_workspace(plan, DEV)
    qp, dop = torch.cat([q, q]), torch.cat([d_o, d_o])
    op, lp = torch.empty_like(qp), torch.empty(4, 500, device=DEV)
    o, lse = torch.empty_like(q), torch.empty(4, 250, device=DEV)
    rows = torch.arange(500, dtype=torch.int32, device=DEV).view(2, 250)
    B.ca_forward(plan, qp, k, v, op, lp, ws)
    assert torch.isinf(lp[:, 249]).all()  # the last row's window begins behind the first part's keys
    B.ca_merge_partials(rows, op, lp, o, lse, op, lp)
    dqp, dq, dk, dv = torch.empty_like(qp), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    B.ca_backward(plan, qp, k, v, op, dop, lp, dqp, dk, dv, ws)
    B.ca_sum_partial_dq(rows, dqp, dq)
    want, far = U.reference(whole, window, 0, q, k, v, d_o, o)
    # (a part's O, and its dQ, are rounded to bf16 once more than the whole's: the bounds count that rounding twice)
    U.check({"o": o, "dq": dq, "dk": dk, "dv": dv}, want, {x: 2 * y for x, y in far.items()}, ("o", "dq", "dk", "dv"))


def test_kernel_times_are_read():
    b = U.batch([800], [(0, 0, 800)], 8, 2, 64)
    tensors = W.make_tensors(b, DEV)
    want = run(b, 100, 0, tensors)
    q, k, v, d_o = tensors
    plan = B.ca_plan(b, window=100)
    plan.profile_enable()
    ws = B.alloc_workspace(plan, DEV)
    got = {n: torch.zeros_like(x) for n, x in want.items()}
    B.ca_forward(plan, q, k, v, got["o"], got["lse"], ws)
    B.ca_backward(plan, q, k, v, got["o"], d_o, got["lse"], got["dq"], got["dk"], got["dv"], ws)
    assert all(t > 0 for t in plan.profile_read().values())
    assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("heads,d", [((4, 2), 64), ((4, 1), 128), ((2, 2), 128)])
@pytest.mark.parametrize("window,sinks", [(37, 0), (37, 5), (100, 70), (1, 0), (5, 129)])
def test_keys_that_nobody_sees_may_hold_anything(window, sinks, heads, d):
    """NaN or Inf in K and V before, between and behind the windows: every result as with finite values there, zero for those keys.  Task 3's
    keys end before its rows' windows, document 2 is seen by nobody without sinks."""
    b = U.batch([700, 300, 200], [(0, 150, 40), (0, 190 + 2 * window, 70), (0, 650, 1), (0, 600, 3), (1, 10, 64), (2, 150, 30)], *heads, d,
                {3: 300, 5: 20}, seed=4)
    q, k, v, d_o = W.make_tensors(b, DEV)
    see = U.visible(b, window, sinks)
    unseen = torch.from_numpy(~see.any(0)).to(DEV)
    assert unseen.sum() > 300
    want = run(b, window, sinks, (q, k, v, d_o))
    check(b, window, sinks, want, (q, k, v, d_o))
    for value in (float("nan"), float("inf"), -float("inf")):
        for both in ("k", "v", "kv"):
            kk, vv = k.clone(), v.clone()
            if "k" in both:
                kk[unseen] = value
            if "v" in both:
                vv[unseen] = value
            got = run(b, window, sinks, (q, kk, vv, d_o))
            for n, x in want.items():
                assert torch.equal(got[n], x), (n, value, both)
    for n in ("dk", "dv"):
        assert not want[n][unseen].any()


def test_tensors_out_of_line_are_refused():
    b = U.batch([300], [(0, 0, 300)], 2, 1, 64)
    tensors = W.make_tensors(b, DEV)
    plan = B.ca_plan(b, window=20)
    q, k, v, d_o = tensors
    o, lse = torch.zeros_like(q), torch.zeros(2, 300, device=DEV)
    ws = torch.empty(plan.workspace_bytes()[1], dtype=torch.uint8, device=DEV)
    B.ca_forward(plan, q, k, v, o, lse, ws)

    def shifted(x):
        return torch.cat([x.new_zeros(1), x.flatten()])[1:].view(x.shape)

    for i in range(4):
        args = [q, k, v, o]
        args[i] = shifted(args[i])
        with pytest.raises(B.CaError) as e:
            B.ca_forward(plan, *args, lse, ws)
        assert e.value.code == B.CA_ERR_INVALID_ARG
    for i in range(8):
        args = [q, k, v, o, d_o, torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]
        args[i] = shifted(args[i])
        with pytest.raises(B.CaError) as e:
            B.ca_backward(plan, *args[:5], lse, *args[5:], ws)
        assert e.value.code == B.CA_ERR_INVALID_ARG
