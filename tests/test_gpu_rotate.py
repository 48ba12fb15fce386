"""Turned and normed queries and keys, and their gradients, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import rotary_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import rotary as R
from paper_2510_18121_amd import workloads as W
from paper_2510_18121_amd.autograd import AttentionServer, row_positions

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def gain_of(d, seed):
    return 1 + 0.3 * rand(d, seed=seed, dtype=torch.float32)


def positions(rows, seed=0):
    p = np.random.default_rng(seed).integers(0, 1 << 20, rows)
    p[:4] = [0, 2 ** 31 - 1, -5, 1][:rows]
    return i32(p)


FORMS = [(128, 128, False), (128, 128, True), (128, 64, False), (128, 16, False), (128, 38, False), (128, 2, True), (64, 64, False), (64, 64, True),
         (64, 32, True), (64, 34, False), (64, 0, False)]


@pytest.mark.parametrize("d,rot,interleaved", FORMS)
@pytest.mark.parametrize("rows,hq,hkv,normed", [(1, 32, 8, True), (2, 1, 1, False), (67, 9, 3, True), (300, 17, 16, True), (40, 33, 1, False)])
def test_both_directions(d, rot, interleaved, rows, hq, hkv, normed):
    r = R.Rotation(d, frequencies=R.frequencies(rot, 5e5), interleaved=interleaved, factor=1.25, device=DEV)
    q, k, dyq, dyk = (rand(rows, h, d, seed=i) for i, h in enumerate((hq, hkv, hq, hkv)))
    qp, kp = positions(rows, 1), positions(rows, 2)
    gq, gk = (gain_of(d, 5), gain_of(d, 6)) if normed else (None, None)
    yq, yk, dq, dk = (torch.full_like(x, float("nan")) for x in (q, k, q, k))
    B.ca_rotate(r, q, k, yq, yk, qp, kp, q_gain=gq, k_gain=gk, eps=1e-3)
    dg = [torch.full((d,), float("nan"), device=DEV) if normed else None for _ in range(2)]
    ws = B.alloc_rotate_workspace(DEV).fill_(0xFF)
    B.ca_rotate_backward(r, q, k, dyq, dyk, dq, dk, qp, kp, q_gain=gq, k_gain=gk, dq_gain=dg[0], dk_gain=dg[1], eps=1e-3, ws=ws)
    for x, dy, y, dx, pos, g, got in ((q, dyq, yq, dq, qp, gq, dg[0]), (k, dyk, yk, dk, kp, gk, dg[1])):
        U.close(y, *U.forward(x, pos, r.frequencies, interleaved, 1.25, g, 1e-3))
        want, want_g, far, far_g = U.backward(x, dy, pos, r.frequencies, interleaved, 1.25, g, 1e-3)
        U.close(dx, want, far, 2.0 ** -18)
        if normed:
            U.close_gain(got, want_g, far_g)


@pytest.mark.parametrize("interleaved,rot", [(False, 64), (True, 64), (False, 22)])
def test_many_rows_of_few_heads_and_of_many(interleaved, rot):
    """Waves that go on with rows further on, and rows that several waves share; queries and keys of different numbers of rows."""
    r = R.Rotation(64, frequencies=R.frequencies(rot), interleaved=interleaved, device=DEV)
    q, k, dyq, dyk = rand(20011, 2, 64), rand(37, 200, 64, seed=1), rand(20011, 2, 64, seed=2), rand(37, 200, 64, seed=3)
    qp, kp, gq = positions(20011), positions(37), gain_of(64, 4)
    yq, yk, dq, dk, dg = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k), torch.empty(64, device=DEV)
    B.ca_rotate(r, q, k, yq, yk, qp, kp, q_gain=gq)
    B.ca_rotate_backward(r, q, None, dyq, dyk, dq, dk, qp, kp, q_gain=gq, dq_gain=dg, ws=B.alloc_rotate_workspace(DEV))
    U.close(yq, *U.forward(q, qp, r.frequencies, interleaved, 1.0, gq))
    U.close(yk, *U.forward(k, kp, r.frequencies, interleaved))
    want, want_g, far, far_g = U.backward(q, dyq, qp, r.frequencies, interleaved, 1.0, gq)
    U.close(dq, want, far, 2.0 ** -18)
    U.close_gain(dg, want_g, far_g)
    want, _, far, _ = U.backward(k, dyk, kp, r.frequencies, interleaved)
    U.close(dk, want, far, 2.0 ** -18)


@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (128, 64, True), (128, 42, False), (64, 64, False), (64, 32, True), (64, 26, False)])
def test_tensors_beyond_the_last_cache(d, rot, interleaved):
    """More than 384 MiB read and written, which passes the caches by: the same bits as in pieces of less."""
    r = R.Rotation(d, frequencies=R.frequencies(rot), interleaved=interleaved, device=DEV)
    rows, heads = 41003, 20 * 128 // d
    q, dy, pos, g = rand(rows, heads, d), rand(rows, heads, d, seed=1), positions(rows), gain_of(d, 2)
    ws = B.alloc_rotate_workspace(DEV)

    def both(a, e):
        y, dx, dg = torch.empty_like(q[a:e]), torch.empty_like(q[a:e]), torch.empty(d, device=DEV)
        B.ca_rotate(r, q[a:e], None, y, None, pos[a:e], q_gain=g)
        B.ca_rotate_backward(r, q[a:e], None, dy[a:e], None, dx, None, pos[a:e], q_gain=g, dq_gain=dg, ws=ws)
        return y, dx, dg

    y, dx, dg = both(0, rows)
    parts = [both(a, min(a + 14000, rows)) for a in range(0, rows, 14000)]
    assert torch.equal(y, torch.cat([p[0] for p in parts])) and torch.equal(dx, torch.cat([p[1] for p in parts]))
    tail = slice(rows - 500, rows)
    U.close(y[tail], *U.forward(q[tail], pos[tail], r.frequencies, interleaved, 1.0, g))
    # (sums of up to 512 terms one after the other here too; the magnitudes of all terms)
    far = U.backward(q[tail], dy[tail], pos[tail], r.frequencies, interleaved, 1.0, g)[3] * (rows / 500) * 1.2
    assert ((dg - sum(p[2] for p in parts)).abs() <= 2.0 ** -14 * far).all()


def test_rows_of_a_joint_projection_and_in_place():
    r = R.Rotation(128, device=DEV)
    joint = rand(50, 6 * 128 + 8)
    before, pos, g = joint.clone(), positions(50), gain_of(128, 1)
    q, k = joint[:, :512].unflatten(1, (4, 128)), joint[:, 512:640].unflatten(1, (1, 128))
    y = torch.full((52, 5, 128), 7.0, device=DEV, dtype=torch.bfloat16)
    yq, yk = y[1:51, :4], y[1:51, 4:]
    B.ca_rotate(r, q, k, yq, yk, pos, q_gain=g, k_gain=g)
    assert torch.equal(joint, before) and (y[0] == 7).all() and (y[51] == 7).all()
    U.close(yq, *U.forward(q, pos, r.frequencies, False, 1.0, g))
    U.close(yk, *U.forward(k, pos, r.frequencies, False, 1.0, g))
    plain = [torch.empty_like(x) for x in (q.contiguous(), k.contiguous())]
    B.ca_rotate(r, q.contiguous(), k.contiguous(), *plain, pos, q_gain=g, k_gain=g)
    assert torch.equal(plain[0], yq) and torch.equal(plain[1], yk)
    B.ca_rotate(r, q, k, q, k, pos, q_gain=g, k_gain=g)
    assert torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(joint[:, 640:], before[:, 640:])


def test_gradients_in_place_and_out_of_a_joint_tensor():
    r = R.Rotation(64, rot_dim=32, interleaved=True, device=DEV)
    joint, d_joint, pos, g = rand(33, 5 * 64), rand(33, 5 * 64, seed=1), positions(33), gain_of(64, 2)
    q, dy = joint[:, 64:192].unflatten(1, (2, 64)), d_joint[:, 64:192].unflatten(1, (2, 64))
    want, want_g, far, far_g = U.backward(q, dy, pos, r.frequencies, True, 1.0, g)
    before, dg = d_joint.clone(), torch.empty(64, device=DEV)
    B.ca_rotate_backward(r, q, None, dy, None, dy, None, pos, q_gain=g, dq_gain=dg, ws=B.alloc_rotate_workspace(DEV))
    U.close(dy, want, far, 2.0 ** -18)
    U.close_gain(dg, want_g, far_g)
    assert torch.equal(d_joint[:, :64], before[:, :64]) and torch.equal(d_joint[:, 192:], before[:, 192:])


def test_rows_beyond_4_gib():
    r = R.Rotation(64, device=DEV)
    far = torch.empty(5, 1 << 30, dtype=torch.bfloat16, device=DEV)  # 8 GiB
    q = far[:, :128].unflatten(1, (2, 64))
    q.copy_(rand(5, 2, 64))
    y, pos = torch.empty(5, 2, 64, dtype=torch.bfloat16, device=DEV), positions(5)
    B.ca_rotate(r, q, None, y, None, pos)
    U.close(y, *U.forward(q, pos, r.frequencies, False))
    z = torch.zeros_like(y)
    B.ca_rotate_backward(r, None, None, y, None, q, None, pos)
    B.ca_rotate_backward(r, None, None, y, None, z, None, pos)
    assert torch.equal(q, z)


@pytest.mark.parametrize("n_seqs", [1, 3, 63, 64, 65, 700, 4096])
def test_positions_of_sequences(n_seqs):
    """As binding.ca_cache_append takes the rows: the last ones of each sequence; rows of none are left as they are."""
    rng = np.random.default_rng(n_seqs)
    n = rng.integers(0, 4, n_seqs)
    n[rng.integers(n_seqs)] = 5
    first, rows = 2, int(n.sum()) + 6  # two rows before the sequences, four behind
    start = first + np.concatenate([[0], np.cumsum(n)])
    lens = n + rng.integers(0, 1 << 20, n_seqs)
    pos = np.concatenate([np.arange(t - m, t) for m, t in zip(n, lens)])
    r, q, k = R.Rotation(128, device=DEV), rand(rows, 3, 128), rand(rows, 1, 128, seed=1)
    yq, yk = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    B.ca_rotate(r, q, k, yq, yk, where=(i32(start), i32(lens), None))
    want = [torch.empty_like(x[first:-4]) for x in (q, k)]
    B.ca_rotate(r, q[first:-4], k[first:-4], *want, i32(pos))
    for y, w in ((yq, want[0]), (yk, want[1])):
        assert torch.equal(y[first:-4], w) and (y[:first] == 5).all() and (y[-4:] == 5).all()
    dx = torch.full_like(q, 5.0)
    B.ca_rotate_backward(r, None, None, q, None, dx, None, where=(i32(start), i32(lens)))
    assert (dx[:first] == 5).all() and (dx[-4:] == 5).all()
    U.close(dx[first:-4], *U.backward(None, q[first:-4], i32(pos), r.frequencies, False)[::2], 2.0 ** -18)


def test_sequences_out_of_range_are_clamped():
    """Rows beyond the tensor count as far as it goes."""
    r, q = R.Rotation(64, device=DEV), rand(6, 1, 64)
    y = torch.full_like(q, 5.0)
    B.ca_rotate(r, q, None, y, None, where=(i32([-3, 4, 100, 2 ** 31 - 1]), i32([50, 60, 70])))
    want = torch.empty_like(q)
    B.ca_rotate(r, q, None, want, None, i32([46, 47, 48, 49, 58, 59]))
    assert torch.equal(y, want)


def test_what_is_not_finite_stays_where_it_is():
    r = R.Rotation(128, rot_dim=64, device=DEV)
    x, pos = rand(4, 8, 128), i32([3, 4, 5, 6])
    clean = torch.empty_like(x)
    B.ca_rotate(r, x, None, clean, None, pos)
    x[1, 2, 100], x[1, 3, 127], x[2, 5, 7] = float("inf"), float("nan"), float("inf")
    y = torch.empty_like(x)
    B.ca_rotate(r, x, None, y, None, pos)
    assert y[1, 2, 100] == float("inf") and torch.isnan(y[1, 3, 127]) and not torch.isfinite(y[2, 5, 7]) and not torch.isfinite(y[2, 5, 39])
    y[1, 2, 100], y[1, 3, 127], y[2, 5, 7], y[2, 5, 39] = clean[1, 2, 100], clean[1, 3, 127], clean[2, 5, 7], clean[2, 5, 39]
    assert torch.equal(y, clean)


def test_a_head_of_zeros():
    r, x, g = R.Rotation(64, device=DEV), torch.zeros(2, 3, 64, dtype=torch.bfloat16, device=DEV), gain_of(64, 1)
    y, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(64, device=DEV)
    B.ca_rotate(r, x, None, y, None, i32([5, 6]), q_gain=g)
    B.ca_rotate_backward(r, x, None, rand(2, 3, 64), None, dx, None, i32([5, 6]), q_gain=g, dq_gain=dg, ws=B.alloc_rotate_workspace(DEV))
    want, _, far, _ = U.backward(x, rand(2, 3, 64), i32([5, 6]), r.frequencies, False, 1.0, g)
    U.close(dx, want, far, 2.0 ** -18)
    assert (y == 0).all() and (dg == 0).all()


def test_gain_gradient_of_no_rows_is_zero():
    r, x = R.Rotation(64, device=DEV), torch.empty(0, 3, 64, dtype=torch.bfloat16, device=DEV)
    dg = torch.full((64,), 5.0, device=DEV)
    B.ca_rotate_backward(r, x, None, x, None, torch.empty_like(x), None, i32([]), q_gain=gain_of(64, 1), dq_gain=dg, ws=B.alloc_rotate_workspace(DEV))
    assert (dg == 0).all()


def test_differentiable_op():
    """Gradients of a joint projection's views and of gains of both types, twice the same bits; a gradient that is an expanded scalar."""
    r = R.Rotation(128, device=DEV)
    pos = positions(70)
    grads = []
    for _ in range(2):
        joint = rand(70, 6 * 128).requires_grad_()
        gq, gk = gain_of(128, 1).requires_grad_(), gain_of(128, 2).to(torch.bfloat16).requires_grad_()
        q, k = joint[:, :512].unflatten(1, (4, 128)), joint[:, 512:].unflatten(1, (2, 128))
        yq, yk = r(q, k, pos, q_gain=gq, k_gain=gk)
        grads.append(torch.autograd.grad(yq.sum() + (yk * yk.detach()).sum(), (joint, gq, gk)))
    assert all(torch.equal(a, b) for a, b in zip(*grads))
    dj, dgq, dgk = grads[0]
    want, want_g, far, far_g = U.backward(q.detach(), torch.ones_like(yq), pos, r.frequencies, False, 1.0, gq.detach())
    U.close(dj[:, :512].unflatten(1, (4, 128)), want, far, 2.0 ** -18)
    U.close_gain(dgq, want_g, far_g)
    want, want_g, far, far_g = U.backward(k.detach(), yk.detach(), pos, r.frequencies, False, 1.0, gk.detach().float())
    U.close(dj[:, 512:].unflatten(1, (2, 128)), want, far, 2.0 ** -18)
    assert dgk.dtype == torch.bfloat16
    assert ((dgk.double() - want_g).abs() <= 2.0 ** -8 * want_g.abs() + 2.0 ** -14 * far_g).all()


def test_gain_gradient_against_differences():
    """y is linear in the gain: the slope of <y, dy> along a direction, with dy = y, whose roundings (2^-9 of each of y's terms at most, unlike signs)
    are far below a hundredth of the sum of squares that it is."""
    r, q, g, pos = R.Rotation(64, device=DEV), rand(40, 4, 64), gain_of(64, 1), positions(40)
    y = [torch.empty_like(q) for _ in range(3)]
    B.ca_rotate(r, q, None, y[0], None, pos, q_gain=g)
    for i, sign in ((1, 1), (2, -1)):
        B.ca_rotate(r, q, None, y[i], None, pos, q_gain=g + 0.5 * sign * g)
    dx, dg = torch.empty_like(q), torch.empty_like(g)
    B.ca_rotate_backward(r, q, None, y[0], None, dx, None, pos, q_gain=g, dq_gain=dg, ws=B.alloc_rotate_workspace(DEV))
    slope = ((y[1].double() - y[2].double()) * y[0].double()).sum()
    assert abs(slope - (dg * g).double().sum()) < 0.01 * slope


def test_second_gradients_are_refused():
    r, q = R.Rotation(64, device=DEV), rand(3, 1, 64).requires_grad_()
    y = r(q, None, i32([1, 2, 3]))
    dq, = torch.autograd.grad(y.float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        dq.sum().backward()


def test_positions_that_change_before_the_backward_are_noticed():
    r, q = R.Rotation(64, device=DEV), rand(3, 1, 64).requires_grad_()
    pos, start, lens = i32([1, 2, 3]), i32([0, 3]), i32([9])
    for y, changed in ((r(q, None, pos), pos), (r(q, None, where=(start, lens)), lens)):
        changed += 1
        with pytest.raises(RuntimeError):
            torch.autograd.grad(y, q, torch.ones_like(y))


def test_gains_that_are_strided_and_frequencies_of_every_kind():
    """A gain out of a larger tensor; slowed frequencies, negative ones, and far positions of them."""
    freq = np.concatenate([R.by_parts(R.frequencies(40, 1e4), 8, 4096), [-0.3, 0.0, 6.5]])
    r = R.Rotation(64, frequencies=freq, factor=0.7, device=DEV)
    q, pos = rand(9, 2, 64), i32([0, 1, 2 ** 31 - 1, -(2 ** 31), 4096, 77777777, -1, 3, 2 ** 30])
    both = torch.stack([gain_of(64, 1), gain_of(64, 2)], 1).requires_grad_()
    y = r(q, None, pos, q_gain=both[:, 1])
    U.close(y.detach(), *U.forward(q, pos, freq, False, 0.7, both[:, 1].detach()))
    dg, = torch.autograd.grad(y, both, torch.ones_like(y))
    _, want, _, far = U.backward(q, torch.ones_like(q), pos, freq, False, 0.7, both[:, 1].detach())
    U.close_gain(dg[:, 1], want, far)
    assert (dg[:, 0] == 0).all()


def test_no_gradient_reaches_rows_of_no_sequence():
    r, q = R.Rotation(64, device=DEV), rand(5, 2, 64).requires_grad_()
    y = r(q, None, where=(i32([1, 4]), i32([9])))
    dq, = torch.autograd.grad(y, q, torch.ones_like(y))
    assert (dq[0] == 0).all() and (dq[4] == 0).all() and (dq[1:4] != 0).any()


def test_graph_and_streams():
    """Captured once, replayed as positions and rows change; and on another stream."""
    r, q, k, g = R.Rotation(128, device=DEV), rand(9, 8, 128), rand(9, 2, 128, seed=1), gain_of(128, 1)
    start, lens = i32([0, 4, 9]), i32([10, 20])
    yq, yk, dq, dg, ws = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty(128, device=DEV), B.alloc_rotate_workspace(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def calls(stream=None):
        B.ca_rotate(r, q, k, yq, yk, where=(start, lens), q_gain=g, k_gain=g, stream=stream)
        B.ca_rotate_backward(r, q, None, yq, None, dq, None, where=(start, lens), q_gain=g, dq_gain=dg, ws=ws, stream=stream)

    calls(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        lens += 100000 * i
        q.copy_(rand(9, 8, 128, seed=10 + i))
        start.copy_(i32([0, 4 + i, 9]))
        for t in (yq, yk, dq, dg):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (yq, yk, dq, dg)]
        calls(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (yq, yk, dq, dg)))
        pos = torch.cat([torch.arange(int(t) - n, int(t)) for n, t in zip((4 + i, 5 - i), lens)]).to(DEV)
        U.close(got[0], *U.forward(q, pos, r.frequencies, False, 1.0, g))


def test_captured_training_pass():
    """Forward and gradients captured once, with gradients asked of autograd for the leaves directly, and replayed as inputs, positions and gains change."""
    r = R.Rotation(64, device=DEV)
    leaves = [rand(50, 4, 64).requires_grad_(), rand(50, 2, 64, seed=1).requires_grad_(), gain_of(64, 2).requires_grad_(), gain_of(64, 3).requires_grad_()]
    pos, dys = positions(50), [rand(50, 4, 64, seed=4), rand(50, 2, 64, seed=5)]

    def train(q, k, gq, gk):
        ys = r(q, k, pos, q_gain=gq, k_gain=gk)
        return *(y.detach() for y in ys), *torch.autograd.grad(ys, (q, k, gq, gk), dys)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train(*leaves)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = train(*leaves)
    for i in range(3):
        with torch.no_grad():
            leaves[0].copy_(rand(50, 4, 64, seed=20 + i)), leaves[2].mul_(1.1)
        pos += 1000
        for t in out:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        want = train(*(t.detach().clone().requires_grad_() for t in leaves))
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("window", [None, 40])
def test_attention_server_with_a_rotation(window):
    """The same bits as turning first; positions are those in the documents, for shards in any order."""
    b = W.custom([200, 90], [(0, 64, 136), (1, 0, 90), (0, 0, 64)], 4, 2, 64, seed=5)
    q, k, v, do = W.make_tensors(b, DEV)
    r = R.Rotation(64, base=5e5, device=DEV)
    gq, gk = gain_of(64, 1), gain_of(64, 2)
    leaves = [t.clone().requires_grad_() for t in (q, k, v, gq, gk)]
    o = AttentionServer(b, DEV, window=window, rotation=r)(*leaves)
    got = torch.autograd.grad(o, leaves, do)
    qp, kp = (torch.from_numpy(x).to(DEV) for x in row_positions(b))
    assert qp.tolist() == list(range(64, 200)) + list(range(90)) + list(range(64))
    again = [t.clone().requires_grad_() for t in (q, k, v, gq, gk)]
    turned = r(*again[:2], qp, kp, q_gain=again[3], k_gain=again[4])
    o2 = AttentionServer(b, DEV, window=window)(*turned, again[2])
    assert torch.equal(o, o2)
    assert all(torch.equal(a, c) for a, c in zip(got, torch.autograd.grad(o2, again, do)))
    # positions count by their differences alone
    far = r(q, k, qp + 500000, kp + 500000, q_gain=gq, k_gain=gk)
    o3 = AttentionServer(b, DEV, window=window)(*far, v)
    assert (o3.double() - o.double()).norm() < 0.01 * o.double().norm()


def test_tensors_that_are_refused():
    r, q, pos = R.Rotation(64, device=DEV), rand(4, 2, 64), i32([0, 1, 2, 3])
    y = torch.empty_like(q)
    for args in ((q[..., :32], None, y, None, pos), (q.float(), None, y, None, pos), (q, None, y[:3], None, pos), (q, None, y, None, pos[:3]),
                 (q, None, y, None, pos.long()), (q, None, y, None), (q.transpose(0, 1), None, y.transpose(0, 1), None, i32([0, 1])), (q.cpu(), None, y, None, pos),
                 (q, None, y, None, pos.cpu())):
        with pytest.raises(ValueError):
            B.ca_rotate(r, *args)
    with pytest.raises(ValueError):
        B.ca_rotate(r, q, None, y, None, pos, q_gain=torch.ones(64, device=DEV, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.ca_rotate_backward(r, None, None, q, None, y, None, pos, q_gain=torch.ones(64, device=DEV), dq_gain=torch.ones(64, device=DEV))
    with pytest.raises(B.CaError):
        B.ca_rotate(r, rand(4 * 128 + 8)[4:-4].view(4, 2, 64), None, y, None, pos)
    with pytest.raises(B.CaError):
        B.ca_rotate_backward(r, q, None, q, None, y, None, pos, q_gain=torch.ones(64, device=DEV), dq_gain=torch.ones(64, device=DEV))
