"""Rows that take no part in a batch, whatever they hold, leave no trace in the gradients of the rotation's gains."""
import numpy as np
import pytest
import torch

import rotary_util as U
import window_util
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import rotary as R
from paper_2510_18121_amd import workloads as W
from paper_2510_18121_amd.autograd import AttentionServer, row_positions
from test_gpu_rotate import DEV, gain_of, i32, positions, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 3)])
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_attention_server_with_rows_of_nobody(window, sinks, eps):
    """Rows of no task and keys of no document, and with a window keys that no row sees, hold NaN, infinities and zeros: the same bits as with ordinary
    numbers there, and the definition's gradients."""
    b = W.custom([200, 90, 130], [(0, 100, 60), (1, 0, 90), (2, 90, 30)], 4, 2, 64, seed=5)
    b.total_q, b.total_kv = b.total_q + 9, b.total_kv + 7
    see = window_util.visible(b, window or 10 ** 9, sinks)
    q, k, v, do = W.make_tensors(b, DEV)
    in_q = see.any(1)
    in_k = see.any(0) if window else np.arange(b.total_kv) < sum((200, 90, 130))
    assert not in_q.all() and not in_k.all()
    r, gq, gk = R.Rotation(64, base=5e5, device=DEV), gain_of(64, 1), gain_of(64, 2)
    server, plain = (AttentionServer(b, DEV, window=window, sinks=sinks, **kw) for kw in ({"rotation": r, "eps": eps}, {}))
    results = []
    for fill in (None, float("nan"), float("inf"), 0.0):
        qx, kx = q.clone(), k.clone()
        if fill is not None:
            qx[torch.from_numpy(~in_q).to(DEV)] = fill
            kx[torch.from_numpy(~in_k).to(DEV)] = fill
        leaves = [t.clone().requires_grad_() for t in (qx, kx, v, gq, gk)]
        o = server(*leaves)
        results.append((o[torch.from_numpy(in_q).to(DEV)], *torch.autograd.grad(o, leaves, do)))
    for other in results[1:]:
        assert all(torch.equal(a, c) for a, c in zip(results[0], other))
    _, dq, dk, _, dgq, dgk = results[0]
    used_k = torch.from_numpy(see.any(0)).to(DEV)
    used_q = torch.from_numpy(in_q).to(DEV)
    assert (dq[~used_q] == 0).all() and (dk[~used_k] == 0).all() and torch.isfinite(dq).all() and torch.isfinite(dk).all()
    qp, kp = (torch.from_numpy(x).to(DEV) for x in row_positions(b))
    turned = [t.detach().requires_grad_() for t in r(q, k, qp, kp, q_gain=gq, k_gain=gk, eps=eps)]
    dys = torch.autograd.grad(plain(*turned, v), turned, do)
    for x, dy, pos, g, used, dx, dg in ((q, dys[0], qp, gq, used_q, dq, dgq), (k, dys[1], kp, gk, used_k, dk, dgk)):
        want, want_g, far, far_g = U.backward(x[used], dy[used], pos[used], r.frequencies, False, 1.0, g, eps)
        U.close(dx[used], want, far, 2.0 ** -18)
        U.close_gain(dg, want_g, far_g)


@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (64, 64, True), (128, 38, False)])
def test_gaps(d, rot, interleaved):
    """Their gradients are left as they are by the call and zero by the differentiable op, forward and the other rows are as without; without gaps
    the position stands for itself."""
    r = R.Rotation(d, frequencies=R.frequencies(rot), interleaved=interleaved, device=DEV)
    q, dy, g, ws = rand(700, 9, d), rand(700, 9, d, seed=1), gain_of(d, 2), B.alloc_rotate_workspace(DEV)
    gap = torch.zeros(700, dtype=torch.bool, device=DEV)
    gap[[0, 1, 5, 699]] = True
    gap[100:300] = True
    pos = positions(700)
    marked = torch.where(gap, R.GAP, pos).int()
    want, want_g, far, far_g = U.backward(q[~gap], dy[~gap], pos[~gap], r.frequencies, interleaved, 1.0, g)
    x = q.clone()
    x[gap] = float("nan")
    dx, dg = torch.full_like(q, 5.0), torch.empty(d, device=DEV)
    B.ca_rotate_backward(r, x, None, dy, None, dx, None, marked, q_gain=g, dq_gain=dg, ws=ws, q_gaps=True)
    assert (dx[gap] == 5).all()
    U.close(dx[~gap], want, far, 2.0 ** -18)
    U.close_gain(dg, want_g, far_g)
    leaf, gain = x.clone().requires_grad_(), g.clone().requires_grad_()
    y = r(leaf, None, pos, q_gain=gain, grad_pos=(marked, None))
    plain = r(q, None, pos, q_gain=g)
    assert torch.equal(y[~gap], plain[~gap])
    got = torch.autograd.grad(y, (leaf, gain), dy)
    assert (got[0][gap] == 0).all() and torch.equal(got[0][~gap], dx[~gap]) and torch.equal(got[1], dg)
    # of keys alone, by the positions of the queries; queries and their gain as without
    leaves = [t.clone().requires_grad_() for t in (q, x, g, g)]
    dq, dk, dgq, dgk = torch.autograd.grad(r(*leaves[:2], pos, q_gain=leaves[2], k_gain=leaves[3], grad_pos=(None, marked)), leaves, (dy, dy))
    assert torch.equal(dk, got[0]) and torch.equal(dgk, dg)
    B.ca_rotate_backward(r, q, None, dy, None, dx, None, pos, q_gain=g, dq_gain=dg, ws=ws)
    assert torch.equal(dq, dx) and torch.equal(dgq, dg)
    first = i32([R.GAP, 3])
    B.ca_rotate_backward(r, q[:2], None, dy[:2], None, dx[:2], None, first, q_gain=g, dq_gain=dg, ws=ws)
    U.close(dx[:2], *U.backward(q[:2], dy[:2], first, r.frequencies, interleaved, 1.0, g)[::2], 2.0 ** -18)
